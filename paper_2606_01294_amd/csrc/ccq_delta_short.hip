// ccq_delta_short.hip -- gradients of the plain gated delta rule for a few tokens, in
// fp32 throughout, token by token.
//
// With u_t = beta_t (v_t - alpha_t S_{t-1} k_t), S_t = alpha_t S_{t-1} + u_t k_t^T and
// o_t = s S_t q_t, and D = dL/dS_t from the tokens behind t, every token does, last first,
//
//   D += s dO_t q_t^T,   du = D k_t,   dv_t = beta_t du,   dbeta_t = du . (v_t - alpha_t S_{t-1} k_t),
//   dq_t = s S_t^T dO_t,   dk_t = D^T u_t - alpha_t beta_t S_{t-1}^T du,
//   dlogalpha_t = alpha_t (<D, S_{t-1}> - beta_t du . S_{t-1} k_t),
//   D <- alpha_t (D - beta_t du k_t^T).
//
// Why beside the chunked backward: a gate's gradient, and with one or two tokens a whole
// dq or dk, is one number for a head.  The bf16 operands of the chunked form leave such a
// number 2^-9 of its terms' sizes off, and where the terms cancel that is much of it:
// over many tokens and heads the norm averages out (3.5e-3 for dbeta), over 1 to 16 of
// them it was 1e-2 to 2.5e-2 now and then.
//
// Rows of S and D (value channels) run through all tokens on their own, one a wave, four
// a workgroup.  The forward recurrence is run again and
// leaves S_{t-1} of every token in the workspace (fp32); what is summed over rows leaves
// as one partial row a workgroup and token, and a second kernel adds those up, over the
// value heads that share a query/key head too, in a fixed order.
// Bound by the latency of a token's chain: product, sum over the wave, update; backward
// also the trip through LDS (64 tokens: 44 us at 64 x 64, 59 at 256 x 256, and 6 for the
// sums; with 16 lanes a row and 16 rows a workgroup 56 and 113).
#include "ccq_device.h"
#include "ccq_kernels.h"
#include "ccq_plain.h"
#include "ccq_pointwise.h"

namespace ccq {

namespace {
constexpr int kThreadsS = 256, kRowsS = 4;
constexpr int kShortLen = 64;  // longest sequence

template <int NV>
__device__ __forceinline__ float dot(const float (&a)[NV], const float (&b)[NV]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) s += a[i] * b[i];
  return s;
}
__device__ __forceinline__ float wave_sum(float x) {
  x = row_sum<16>(x);
  x += __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, x), 0x401F));
  return x + __shfl_xor(x, 32);
}
}  // namespace

// LEN: the longest sequence that its arrays in LDS hold.
template <int DK, int LEN>
__global__ __launch_bounds__(kThreadsS) void delta_short_kernel(const DeltaShortArgs a) {
  typedef bf16_t T;
  constexpr int NV = DK / 64;  // a lane's channels: NV l ..
  typedef VecN<T, NV> VT;
  typedef VecN<float, NV> VF;
  // the sequence's q and k rows, these rows' v and dO, the gates: one trip to memory
  __shared__ __align__(16) T sq_[LEN][DK], sk[LEN][DK];
  __shared__ T sv[LEN][kRowsS], so[LEN][kRowsS];
  __shared__ float sa[LEN], sb[LEN];
  __shared__ __align__(16) float sum[2][2][kRowsS][DK];  // token parity, dq and dk, row
  __shared__ float gate[2][kRowsS][2];                   // dlogalpha, dbeta
  const int nb = a.dv / kRowsS;
  const int l = lane_id(), w = wave_id();
  const int bh = blockIdx.x / nb, vb = blockIdx.x % nb, r = vb * kRowsS + w;
  const int b = bh / a.HV, h = bh % a.HV;
  const KeyHead kh = key_head(a.HK, a.HV, h);
  const Seq sq = seq_of(a.cu, b, a.T);
  const T* const q0 = static_cast<const T*>(a.q) + seq_off(sq, 0, kh.h, kh.H, DK);
  const T* const k0 = static_cast<const T*>(a.k) + seq_off(sq, 0, kh.h, kh.H, DK);
  const T* const v0 = static_cast<const T*>(a.v) + seq_off(sq, 0, h, a.HV, a.dv) + vb * kRowsS;
  const T* const o0 = static_cast<const T*>(a.dO) + seq_off(sq, 0, h, a.HV, a.dv) + vb * kRowsS;
  T* const dv0 = static_cast<T*>(a.dv_out) + seq_off(sq, 0, h, a.HV, a.dv) + r;
  const size_t qs = (size_t)kh.H * DK, vs = (size_t)a.HV * a.dv;
  const size_t g0 = seq_idx(sq, 0, h, a.HV);
  for (int i = threadIdx.x; i < sq.len * (DK / 8); i += kThreadsS) {
    const int t = i / (DK / 8), c = i % (DK / 8) * 8;
    *reinterpret_cast<bf16x8*>(&sq_[t][c]) = *reinterpret_cast<const bf16x8*>(q0 + t * qs + c);
    *reinterpret_cast<bf16x8*>(&sk[t][c]) = *reinterpret_cast<const bf16x8*>(k0 + t * qs + c);
  }
  for (int i = threadIdx.x; i < sq.len * kRowsS; i += kThreadsS) {
    const int t = i / kRowsS, c = i % kRowsS;
    sv[t][c] = v0[t * vs + c];
    so[t][c] = o0[t * vs + c];
  }
  for (int t = threadIdx.x; t < sq.len; t += kThreadsS) {
    sa[t] = __expf(a.logalpha[g0 + (size_t)t * a.HV]);
    sb[t] = a.beta[g0 + (size_t)t * a.HV];
  }
  // S_{t-1} of token t, this row: the same lane writes and reads it
  float* const hist = a.hist + ((size_t)bh * a.T * a.dv + r) * DK + NV * l;
  const size_t hs = (size_t)a.dv * DK;
  float x[NV], D[NV];
  typename VF::raw nx = {};
  if (a.S0) nx = VF::load(a.S0 + ((size_t)bh * a.dv + r) * DK + NV * l);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    x[i] = nx[i];
    D[i] = 0.f;
  }
  auto row = [&](float(&y)[NV], const T* p) {
    const auto v = VT::load(p + NV * l);
#pragma unroll
    for (int i = 0; i < NV; ++i) y[i] = VT::get(v, i);
  };
  __syncthreads();
  for (int t = 0; t < sq.len; ++t) {
    float k[NV];
    row(k, sk[t]);
    VF::store(hist + t * hs, x);
    const float al = sa[t], u = sb[t] * (f32(sv[t][w]) - al * wave_sum(dot<NV>(x, k)));
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i] = al * x[i] + u * k[i];
  }

  // backward: the state of the token before is requested a token ahead
  if (sq.len > 0) nx = VF::load(hist + (sq.len - 1) * hs);
  for (int t = sq.len - 1; t >= 0; --t) {
    float q[NV], k[NV];
    row(q, sq_[t]);
    row(k, sk[t]);
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i] = nx[i];
    nx = VF::load(hist + (t > 0 ? t - 1 : 0) * hs);
    const float al = sa[t], be = sb[t], wt = a.scale * f32(so[t][w]);
#pragma unroll
    for (int i = 0; i < NV; ++i) D[i] += wt * q[i];
    const float y = wave_sum(dot<NV>(x, k)), du = wave_sum(dot<NV>(D, k)), ds = wave_sum(dot<NV>(D, x));
    const float e = f32(sv[t][w]) - al * y, u = be * e, bd = be * du;
    float pq[NV], pk[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      pq[i] = wt * (al * x[i] + u * k[i]);
      pk[i] = u * D[i] - (al * bd) * x[i];
      D[i] = al * (D[i] - bd * k[i]);
    }
    VF::store(&sum[t & 1][0][w][NV * l], pq);
    VF::store(&sum[t & 1][1][w][NV * l], pk);
    if (l == 0) {
      gate[t & 1][w][0] = al * (ds - bd * y);
      gate[t & 1][w][1] = du * e;
      dv0[t * vs] = to<T>(bd);
    }
    lds_barrier();  // (the other parity's arrays are free behind it)
    const size_t part = ((size_t)bh * a.T + t) * nb + vb;
    for (int c = threadIdx.x; c < 2 * DK; c += kThreadsS) {
      const float(*const in)[DK] = sum[t & 1][c / DK];
      const int ch = c % DK;
      a.part[part * 2 * DK + c] = (in[0][ch] + in[1][ch]) + (in[2][ch] + in[3][ch]);
    }
    if (threadIdx.x < 2) {
      const int m = threadIdx.x;
      a.gpart[part * 2 + m] = (gate[t & 1][0][m] + gate[t & 1][1][m]) + (gate[t & 1][2][m] + gate[t & 1][3][m]);
    }
  }
}

// The partial rows of one token added up: workgroup blockIdx.x is token blockIdx.x % T
// of sequence blockIdx.x / T.
template <typename T>
__global__ __launch_bounds__(kThreadsS) void delta_short_sum_kernel(const DeltaShortArgs a) {
  const int b = blockIdx.x / a.T, t = blockIdx.x % a.T;
  const Seq sq = seq_of(a.cu, b, a.T);
  if (t >= sq.len) return;
  const int nb = a.dv / kRowsS, G = a.HV / a.HK, n = a.HK * a.dk;
  for (int c = threadIdx.x; c < 2 * n; c += kThreadsS) {
    const int m = c / n, hk = (c % n) / a.dk, ch = c % a.dk;
    float s = 0.f;
    for (int g = 0; g < G; ++g) {
      const float* p = a.part + (((size_t)(b * a.HV + hk * G + g) * a.T + t) * nb * 2 + m) * a.dk + ch;
#pragma unroll 16
      for (int i = 0; i < nb; ++i) s += p[(size_t)i * 2 * a.dk];
    }
    static_cast<T*>(m ? a.dk_out : a.dq_out)[seq_off(sq, t, hk, a.HK, a.dk) + ch] = to<T>(s);
  }
  for (int c = threadIdx.x; c < 2 * a.HV; c += kThreadsS) {
    const int h = c >> 1, m = c & 1;
    const float* p = a.gpart + ((size_t)(b * a.HV + h) * a.T + t) * nb * 2 + m;
    float s = 0.f;
#pragma unroll 16
    for (int i = 0; i < nb; ++i) s += p[2 * i];
    static_cast<T*>(m ? a.dbeta_io : a.dla_io)[seq_idx(sq, t, h, a.HV)] = to<T>(s);
  }
}

// Up to 64 tokens a sequence (of the bound on the lengths), 128 tokens times value heads:
// there the chunked form's norms do not average its errors out (64 x 1: up to 4.9e-3 over
// 24 draws, 2.1e-3 here; beyond, with 130 to 136 numbers, 4.7e-3 at most over 64 draws at
// each of eight lengths, 4e-3 for nine in ten), and its seven launches cost as much
// (whole calls with o, 64 x 64 and 256 x 256: 27 and 30 us for one token here; 64 tokens
// of 2 heads 59 and 90, the chunked form 39 and 61; 16 of 8 heads 32 and 75, chunked 35
// and 55).
bool delta_short(int B, int T, int HV, bool is_bf16) {
  return is_bf16 && T <= kShortLen && (long long)B * T * HV <= 128;
}

// Workspace, in floats: the states, the partial rows, the gates' partial sums.
size_t delta_short_hist(int B, int T, int HV, int dk, int dv) { return (size_t)B * T * HV * dv * dk; }
size_t delta_short_part(int B, int T, int HV, int dk, int dv) { return (size_t)B * T * HV * (dv / kRowsS) * 2 * dk; }
size_t delta_short_gpart(int B, int T, int HV, int dv) { return (size_t)B * T * HV * (dv / kRowsS) * 2; }

namespace {
// Short ones hold little LDS, so that four or more workgroups share a compute unit where
// there are many (128 heads of 256 x 256, one token each, whole call: 99 us, with the
// arrays for 64 tokens 150).
template <int DK>
void run_delta_short(const DeltaShortArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.B * a.HV * (a.dv / kRowsS))), block(kThreadsS);
  if (a.T <= 16) hipLaunchKernelGGL((delta_short_kernel<DK, 16>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((delta_short_kernel<DK, kShortLen>), grid, block, 0, st, a);
}
}  // namespace

hipError_t launch_delta_short(const DeltaShortArgs& a, hipStream_t st) {
  switch (a.dk) {
    case 64: run_delta_short<64>(a, st); break;
    case 128: run_delta_short<128>(a, st); break;
    case 256: run_delta_short<256>(a, st); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}
hipError_t launch_delta_short_sum(const DeltaShortArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(delta_short_sum_kernel<bf16_t>, dim3((unsigned)(a.B * a.T)), dim3(kThreadsS), 0, st, a);
  return hipGetLastError();
}

}  // namespace ccq
