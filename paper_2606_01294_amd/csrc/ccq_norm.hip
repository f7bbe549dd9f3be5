// ccq_norm.hip -- group norm of the mixer's head outputs with an activation,
// channels last: forward and backward.
//
// x is [rows, G, D]: a token's G heads of D channels, each normalised on its own
// (an item; statistics over tokens would look ahead).  With n the normalisation,
//   group  n = (x - m) r,  m = mean x,  r = (mean (x - m)^2 + eps)^-1/2
//   rms    n = x r,        r = (mean x^2 + eps)^-1/2
//   l2     n = x r,        r = (sum x^2 + eps)^-1/2
//   z = n w + b,   y = z act(gate)  with a gate,  y = act(z)  without.
// Backward, with c = 1 / D (1 for l2) and h = dz w:
//   dz = dy act(gate), dgate = dy z act'(gate)   or   dz = dy act'(z);
//   dw = sum dz n,  db = sum dz;  dx = r (h - [group: mean h] - n c sum(h n)).
//
// Both directions read every tensor once and keep an item in registers between
// its sums and its use, so HBM bounds them.  An item is held by LPI consecutive
// lanes (a power of two, up to a wave; a workgroup above 1024 channels), NV vectors
// of eight channels each.  A slot of LPI lanes takes one head of the rows r, r +
// step, ..: its weights are read once, and the backward sums dw and db in registers
// over all of its rows.  Forward, consecutive slots take consecutive heads (whole
// rows are read); backward, a workgroup's slots take the same head of different rows,
// so that its sums meet in LDS and it leaves one row of partial sums, which a second
// kernel adds up in a fixed order: no atomics, the same bits every time.
// Sums, statistics and the affine part are fp32; what is stored is rounded once.
//
// 16,384 tokens of 8 heads of 256, bf16, gated: forward 43 us (201 MB, 4.6 TB/s; a copy
// of that size from memory runs at 5.1), backward 65 us (335 MB, 5.1 TB/s) and 5 us
// for the partial rows; 4099 rows of 5 heads of 96, fp32: 10 and 4 us, launches and the
// latency of two turns.
#include "ccq_device.h"
#include "ccq_kernels.h"
#include "ccq_pointwise.h"

namespace ccq {

namespace {
constexpr int kNormThreads = 256;

// Sum over the LPI lanes (or, for LPI = 256, the workgroup) that hold an item.
template <int LPI>
__device__ __forceinline__ float item_sum(float x, float* red) {
  x = row_sum<LPI < 16 ? LPI : 16>(x);
  if constexpr (LPI >= 32) x += __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, x), 0x401F));
  if constexpr (LPI >= 64) x += __shfl_xor(x, 32);
  if constexpr (LPI > 64) {  // four waves; the array is free again after the second barrier
    if (lane_id() == 0) red[wave_id()] = x;
    __syncthreads();
    x = (red[0] + red[1]) + (red[2] + red[3]);
    __syncthreads();
  }
  return x;
}

// The lane's channels of one item: vector u is channels 8 (j + LPI u) ..
template <int LPI, int NV>
struct ItemCols {
  int j, nvec;  // lane within the item, vectors per item
  __device__ __forceinline__ bool has(int u) const { return j + LPI * u < nvec; }
  __device__ __forceinline__ int col(int u) const { return 8 * (j + LPI * u); }
};

// n and r of one item, in place of x.
template <int LPI, int NV>
__device__ __forceinline__ float normalise(float (&x)[NV][8], const ItemCols<LPI, NV>& ic, const NormArgs& a, float* red) {
  const float inv = 1.f / (float)a.D;
  if (a.kind == kNormGroup) {
    float s = 0.f;
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += x[u][e];
    const float m = item_sum<LPI>(s, red) * inv;
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[u][e] = ic.has(u) ? x[u][e] - m : 0.f;
  }
  float s = 0.f;
#pragma unroll
  for (int u = 0; u < NV; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += x[u][e] * x[u][e];
  s = item_sum<LPI>(s, red);
  const float r = 1.f / sqrtf(s * (a.kind == kNormL2 ? 1.f : inv) + a.eps);
#pragma unroll
  for (int u = 0; u < NV; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[u][e] *= r;
  return r;
}

template <int LPI, int NV>
__device__ __forceinline__ void load_affine(float (&w)[NV][8], const float* p, int head, float other, const ItemCols<LPI, NV>& ic,
                                            const NormArgs& a) {
  const float* q = p + (a.shared ? 0 : (size_t)head * a.D);
#pragma unroll
  for (int u = 0; u < NV; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) w[u][e] = p && ic.has(u) ? q[ic.col(u) + e] : other;
}
}  // namespace

template <typename T, int LPI, int NV, bool GATE>
__global__ __launch_bounds__(kNormThreads) void norm_fwd_kernel(const NormArgs a) {
  typedef Vec8<T> V;
  constexpr int U = NV == 1 ? 2 : 1;  // items in flight
  __shared__ float red[4];
  const long long s = ((long long)blockIdx.x * kNormThreads + threadIdx.x) / LPI;
  if (s >= a.slots) return;  // whole slots (LPI = 256: the workgroup)
  const ItemCols<LPI, NV> ic{(int)(threadIdx.x % LPI), a.D / 8};
  const int head = (int)(s % a.G);
  const long long step = a.slots / a.G;
  const T* x = static_cast<const T*>(a.x) + (size_t)head * a.D;
  const T* gate = static_cast<const T*>(a.gate) + (size_t)head * a.D;
  T* y = static_cast<T*>(a.y) + (size_t)head * a.D;
  float w[NV][8], b[NV][8];
  load_affine(w, a.w, head, 1.f, ic, a);
  load_affine(b, a.bias, head, 0.f, ic, a);
  for (long long row = s / a.G; row < a.rows; row += U * step) {
    typename V::raw rx[U][NV], rg[U][NV];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const long long rr = row + i * step < a.rows ? row + i * step : row;
#pragma unroll
      for (int u = 0; u < NV; ++u)
        if (ic.has(u)) {
          rx[i][u] = V::load(x + (size_t)rr * a.ldx + ic.col(u));
          if constexpr (GATE) rg[i][u] = V::load(gate + (size_t)rr * a.ldg + ic.col(u));
        }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const long long rr = row + i * step;
      if (rr >= a.rows) break;
      float v[NV][8];
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[u][e] = ic.has(u) ? V::get(rx[i][u], e) : 0.f;
      normalise<LPI, NV>(v, ic, a, red);
#pragma unroll
      for (int u = 0; u < NV; ++u)
        if (ic.has(u)) {
          float o[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float z = v[u][e] * w[u][e] + b[u][e];
            if constexpr (GATE) o[e] = z * Act<T>::value(a.act, V::get(rg[i][u], e));
            else o[e] = Act<T>::value(a.act, z);
          }
          V::store(y + (size_t)rr * a.G * a.D + ic.col(u), o);
        }
    }
  }
}

// Workgroup: head blockIdx.x % G, its slots the rows r, r + 1, .. of row block
// blockIdx.x / G.  Its sums go to partial row blockIdx.x / G, columns head D + ..
// (with one weight for all heads: to a row of their own, columns 0 ..), db behind
// all of dw.
template <typename T, int LPI, int NV, bool GATE>
__global__ __launch_bounds__(kNormThreads) void norm_bwd_kernel(const NormArgs a) {
  typedef Vec8<T> V;
  constexpr int SPB = kNormThreads / LPI;  // slots per workgroup
  __shared__ float red[4];
  const ItemCols<LPI, NV> ic{(int)(threadIdx.x % LPI), a.D / 8};
  const unsigned rb = blockIdx.x / a.G;
  const int head = blockIdx.x - rb * a.G;
  const long long step = a.slots / a.G;
  const T* x = static_cast<const T*>(a.x) + (size_t)head * a.D;
  const T* gate = static_cast<const T*>(a.gate) + (size_t)head * a.D;
  const T* dy = static_cast<const T*>(a.dy) + (size_t)head * a.D;
  T* dx = static_cast<T*>(a.dx) + (size_t)head * a.D;
  T* dgate = static_cast<T*>(a.dgate) + (size_t)head * a.D;
  const size_t ldy = (size_t)a.G * a.D;
  const float c = a.kind == kNormL2 ? 1.f : 1.f / (float)a.D;
  float w[NV][8], b[NV][8], dw[NV][8], db[NV][8];
  load_affine(w, a.w, head, 1.f, ic, a);
  load_affine(b, a.bias, head, 0.f, ic, a);
#pragma unroll
  for (int u = 0; u < NV; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[u][e] = db[u][e] = 0.f;

  // the next item's tensors are requested while one is worked on
  typename V::raw rx[NV], rg[NV], rd[NV];
  auto load = [&](long long row) {
#pragma unroll
    for (int u = 0; u < NV; ++u)
      if (ic.has(u)) {
        rx[u] = V::load(x + (size_t)row * a.ldx + ic.col(u));
        if constexpr (GATE) rg[u] = V::load(gate + (size_t)row * a.ldg + ic.col(u));
        rd[u] = V::load(dy + (size_t)row * ldy + ic.col(u));
      }
  };
  const long long first = (long long)rb * SPB + threadIdx.x / LPI;
  if (first < a.rows) load(first);
  for (long long row = first; row < a.rows; row += step) {
    float n[NV][8], g[NV][8], d[NV][8];
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        n[u][e] = ic.has(u) ? V::get(rx[u], e) : 0.f;
        if constexpr (GATE) g[u][e] = ic.has(u) ? V::get(rg[u], e) : 0.f;
        d[u][e] = ic.has(u) ? V::get(rd[u], e) : 0.f;
      }
    if (row + step < a.rows) load(row + step);
    const float r = normalise<LPI, NV>(n, ic, a, red);
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      float og[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float z = n[u][e] * w[u][e] + b[u][e];
        float av, ad;
        Act<T>::both(a.act, GATE ? g[u][e] : z, av, ad);
        float dz;
        if constexpr (GATE) {
          og[e] = d[u][e] * z * ad;
          dz = d[u][e] * av;
        } else {
          dz = d[u][e] * ad;
        }
        dw[u][e] += dz * n[u][e];
        db[u][e] += dz;
        const float h = dz * w[u][e];
        d[u][e] = h;
        s0 += h;
        s1 += h * n[u][e];
      }
      if constexpr (GATE)
        if (ic.has(u)) V::store(dgate + (size_t)row * ldy + ic.col(u), og);
    }
    s1 = item_sum<LPI>(s1, red) * c;
    s0 = a.kind == kNormGroup ? item_sum<LPI>(s0, red) * c : 0.f;
#pragma unroll
    for (int u = 0; u < NV; ++u)
      if (ic.has(u)) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = r * (d[u][e] - s0 - n[u][e] * s1);
        V::store(dx + (size_t)row * ldy + ic.col(u), o);
      }
  }

  if (!a.part) return;
  const bool bias = a.bias != nullptr;
  const size_t cols = (size_t)(a.shared ? 1 : a.G) * a.D;  // of dw
  const size_t pitch = cols * (bias ? 2 : 1);
  // every slot's sums to LDS, then a column's over the slots in order
  __shared__ __align__(16) float buf[2][LPI > 64 ? 1 : SPB][LPI > 64 ? 4 : LPI * NV * 8];
  float* out = a.part + (a.shared ? (size_t)blockIdx.x * pitch : (size_t)rb * pitch + (size_t)head * a.D);
#pragma unroll
  for (int u = 0; u < NV; ++u)
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const f32x4 w4 = {dw[u][e], dw[u][e + 1], dw[u][e + 2], dw[u][e + 3]};
      const f32x4 b4 = {db[u][e], db[u][e + 1], db[u][e + 2], db[u][e + 3]};
      if constexpr (LPI > 64) {
        if (ic.has(u)) {
          *reinterpret_cast<f32x4*>(out + ic.col(u) + e) = w4;
          if (bias) *reinterpret_cast<f32x4*>(out + cols + ic.col(u) + e) = b4;
        }
      } else {
        *reinterpret_cast<f32x4*>(&buf[0][threadIdx.x / LPI][ic.col(u) + e]) = w4;
        if (bias) *reinterpret_cast<f32x4*>(&buf[1][threadIdx.x / LPI][ic.col(u) + e]) = b4;
      }
    }
  if constexpr (LPI <= 64) {
    __syncthreads();
    for (int i = threadIdx.x; i < a.D; i += kNormThreads)
      for (int q = 0; q < (bias ? 2 : 1); ++q) {
        float t[4] = {};
#pragma unroll
        for (int k = 0; k < SPB; ++k) t[k % 4] += buf[q][k][i];
        out[q * cols + i] = (t[0] + t[1]) + (t[2] + t[3]);
      }
  }
}

namespace {
int norm_lanes(int D) {  // lanes that hold an item: 8 channels each, a power of two
  const int nvec = D / 8;
  int l = 1;
  while (l < nvec && l < 64) l *= 2;
  return nvec > 128 ? 256 : l;
}

// Slots, a multiple of G.  Forward: enough for 32 waves a compute unit and no more,
// so that a slot's weights serve many rows.
long long norm_slots(long long rows, int G, int lanes) {
  long long step = (256ll * 32 * 64 / lanes + G - 1) / G;
  if (step < 1) step = 1;
  return (rows < step ? rows : step) * G;
}
// Backward: row blocks of SPB rows at a time for each head, at most 4 workgroups a
// compute unit in all (what its registers admit), and no more than make every block
// take as many turns (4099 rows of 5 heads of 96, fp32: 129 blocks of two turns 14 us,
// 205 of one or two 16).
long long norm_row_blocks(long long rows, int G, int lanes) {
  const long long spb = kNormThreads / lanes;
  const long long most = (1024 + G - 1) / G, need = (rows + spb - 1) / spb;
  const long long turns = need > 0 ? (need + most - 1) / most : 1;
  return (need + turns - 1) / turns;
}
template <typename T, int LPI, int NV>
hipError_t run_norm(const NormArgs& a, bool bwd, hipStream_t st) {
  const long long nblk = bwd ? norm_row_blocks(a.rows, a.G, LPI) * a.G : (a.slots * LPI + kNormThreads - 1) / kNormThreads;
  const dim3 grid((unsigned)nblk), block(kNormThreads);
  if (!bwd) {
    if (a.gate) hipLaunchKernelGGL((norm_fwd_kernel<T, LPI, NV, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((norm_fwd_kernel<T, LPI, NV, false>), grid, block, 0, st, a);
  } else {
    if (a.gate) hipLaunchKernelGGL((norm_bwd_kernel<T, LPI, NV, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((norm_bwd_kernel<T, LPI, NV, false>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t norm_dispatch(const NormArgs& a, bool bwd, hipStream_t st) {
  switch (norm_lanes(a.D)) {
    case 1: return run_norm<T, 1, 1>(a, bwd, st);
    case 2: return run_norm<T, 2, 1>(a, bwd, st);
    case 4: return run_norm<T, 4, 1>(a, bwd, st);
    case 8: return run_norm<T, 8, 1>(a, bwd, st);
    case 16: return run_norm<T, 16, 1>(a, bwd, st);
    case 32: return run_norm<T, 32, 1>(a, bwd, st);
    case 64:
      if (a.D <= 512) return run_norm<T, 64, 1>(a, bwd, st);
      return run_norm<T, 64, 2>(a, bwd, st);
    case 256:
      if (a.D <= 2048) return run_norm<T, 256, 1>(a, bwd, st);
      if (a.D <= 4096) return run_norm<T, 256, 2>(a, bwd, st);
      return run_norm<T, 256, 4>(a, bwd, st);
  }
  return hipErrorInvalidValue;
}
}  // namespace

bool norm_supported(int D) { return D >= 8 && D <= 8192 && D % 8 == 0; }

// Rows of partial sums of dw (and db) that the backward leaves for colsum.
long long norm_part_rows(long long rows, int G, int D, int shared) {
  return norm_row_blocks(rows, G, norm_lanes(D)) * (shared ? G : 1);
}

hipError_t launch_norm(NormArgs a, bool is_bf16, bool bwd, hipStream_t st) {
  const int lanes = norm_lanes(a.D);
  a.slots = bwd ? norm_row_blocks(a.rows, a.G, lanes) * (kNormThreads / lanes) * a.G : norm_slots(a.rows, a.G, lanes);
  return is_bf16 ? norm_dispatch<bf16_t>(a, bwd, st) : norm_dispatch<float>(a, bwd, st);
}

}  // namespace ccq
