// ccq_conv.hip -- short causal convolution of every channel on its own, with an
// activation: forward, backward and the one-token step.
//
//   z_t = b + sum_{j<W} w_j x_{t-W+1+j},   y_t = act(z_t),
// where x at the W - 1 positions before a sequence's first token is its initial
// state (or zero).  Backward, with dz = dy act'(z) (z formed again) and dz = 0
// behind the last token:
//   dx_p = sum_{i<W} w_{W-1-i} dz_{p+i}     (p < 0: the initial state's gradient),
//   dw_j = sum_t dz_t x_{t-W+1+j},   db = sum_t dz_t.
//
// HBM bounds all three: x (and dy) are read and y (dx) written once.  A lane owns
// a vector of channels and walks a run of consecutive tokens with the window of
// the last W inputs in registers, so a row is read again only by the next run's
// W - 1 tokens of overlap (from cache).  The rows of a batch are requested
// together.  The backward's dw and db are summed in registers over a run, over the
// four runs of a workgroup through LDS, and over the workgroups by a second kernel
// in a fixed order.
// Products and sums are fp32; y and dx are rounded once.
//
// 16,384 tokens of 6144 channels, bf16, W = 4: forward 85 us (403 MB, 4.7 TB/s),
// backward 127 us (604 MB, 4.75 TB/s) and 12 for the partial rows; 8 packed sequences of up
// to 2048 tokens, 2048 channels: backward 39 us (149 MB, 3.8 TB/s) and 5 for the partial
// rows; the same tokens at one length 35 and 4.5, so that 4 of it is the runs behind the
// sequences' ends (three workgroups a compute unit have work in either form, one turn).
// Between events (42 us), runs of 16 or 64 tokens took 44 and 46 us there, eight channels
// a lane 45, eight rows at a time 51; forward, runs of 16 or 64 tokens 90 and 91 us, four
// rows at a time 95.
#include "ccq_device.h"
#include "ccq_kernels.h"
#include "ccq_pointwise.h"

namespace ccq {

namespace {
constexpr int kConvThreads = 256;
constexpr int kConvRun = 32;   // tokens per lane, forward
constexpr int kConvRunB = 32;  // backward

// The taps of VE channels: w[c][j], consecutive in memory, 16-byte loads.
template <int W, int VE>
__device__ __forceinline__ void load_taps(float (&w)[W][VE], const float* p) {
  float flat[W * VE];
#pragma unroll
  for (int i = 0; i < W * VE / 4; ++i) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + 4 * i);
#pragma unroll
    for (int e = 0; e < 4; ++e) flat[4 * i + e] = v[e];
  }
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int e = 0; e < VE; ++e) w[j][e] = flat[e * W + j];
}
template <int VE>
__device__ __forceinline__ void load_bias(float (&b)[VE], const float* p, int c) {
#pragma unroll
  for (int e = 0; e < VE; ++e) b[e] = p ? p[c + e] : 0.f;
}
}  // namespace

template <typename T, int W, int VE, int ACT>
__global__ __launch_bounds__(kConvThreads) void conv_fwd_kernel(const ConvArgs a) {
  typedef VecN<T, VE> V;
  constexpr int NB = 8;  // rows requested together
  const int CV = a.C / VE;
  const unsigned id = blockIdx.x * kConvThreads + threadIdx.x;
  const unsigned rr = id / CV;  // run, over all sequences
  if (rr >= (unsigned)(a.B * a.runs)) return;
  const int c = (int)(id - rr * CV) * VE;
  const int b = rr / a.runs, run = rr - b * a.runs;
  const Seq sq = seq_of(a.cu, b, a.T);
  const int t0 = run * kConvRun;
  if (run > 0 && t0 >= sq.len) return;
  const int t1 = min(t0 + kConvRun, sq.len);
  const T* x = static_cast<const T*>(a.x) + (size_t)sq.row0 * a.ldx + c;
  const T* s0 = static_cast<const T*>(a.state0) + (size_t)b * (W - 1) * a.C + c;
  T* y = static_cast<T*>(a.y) + (size_t)sq.row0 * a.C + c;
  float w[W][VE], bias[VE], win[W][VE];
  load_taps<W, VE>(w, a.w + (size_t)c * W);
  load_bias<VE>(bias, a.bias, c);
  // row p of the sequence, from the initial state where p < 0
  auto row = [&](int p, float (&v)[VE]) {
    if (p >= 0) {
      const auto r = V::load(x + (size_t)p * a.ldx);
#pragma unroll
      for (int e = 0; e < VE; ++e) v[e] = V::get(r, e);
    } else if (a.state0) {
      const auto r = V::load(s0 + (size_t)(p + W - 1) * a.C);
#pragma unroll
      for (int e = 0; e < VE; ++e) v[e] = V::get(r, e);
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) v[e] = 0.f;
    }
  };
#pragma unroll
  for (int j = 0; j < W - 1; ++j) row(t0 - (W - 1) + j, win[j + 1]);

  for (int tb = t0; tb < t1; tb += NB) {
    typename V::raw r[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) r[i] = V::load(x + (size_t)min(tb + i, t1 - 1) * a.ldx);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
#pragma unroll
        for (int e = 0; e < VE; ++e) win[j][e] = win[j + 1][e];
      float o[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        win[W - 1][e] = V::get(r[i], e);
        float z = bias[e];
#pragma unroll
        for (int j = 0; j < W; ++j) z += w[j][e] * win[j][e];
        o[e] = Act<T>::value(ACT, z);
      }
      if (tb + i < t1) V::store(y + (size_t)(tb + i) * a.C, o);
    }
  }
  // the last run (or the only one of an empty sequence) leaves the final state,
  // the last W - 1 inputs
  if (a.stateT && t1 == sq.len) {
    T* sT = static_cast<T*>(a.stateT) + (size_t)b * (W - 1) * a.C + c;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      float v[VE];
      row(sq.len - (W - 1) + j, v);
      V::store(sT + (size_t)j * a.C, v);
    }
  }
}

// One token per sequence: x [B, C], the state [B, W - 1, C] moved on in place.
template <typename T, int W, int VE>
__global__ __launch_bounds__(kConvThreads) void conv_step_kernel(const ConvArgs a) {
  typedef VecN<T, VE> V;
  const int CV = a.C / VE;
  const unsigned id = blockIdx.x * kConvThreads + threadIdx.x;
  const unsigned b = id / CV;
  if (b >= (unsigned)a.B) return;
  const int c = (int)(id - b * CV) * VE;
  T* st = static_cast<T*>(a.stateT) + (size_t)b * (W - 1) * a.C + c;
  typename V::raw r[W];
#pragma unroll
  for (int j = 0; j < W - 1; ++j) r[j] = V::load(st + (size_t)j * a.C);
  r[W - 1] = V::load(static_cast<const T*>(a.x) + (size_t)b * a.ldx + c);
  float w[W][VE], o[VE];
  load_taps<W, VE>(w, a.w + (size_t)c * W);
  load_bias<VE>(o, a.bias, c);
#pragma unroll
  for (int e = 0; e < VE; ++e) {
#pragma unroll
    for (int j = 0; j < W; ++j) o[e] += w[j][e] * V::get(r[j], e);
    o[e] = Act<T>::value(a.act, o[e]);
  }
  V::store(static_cast<T*>(a.y) + (size_t)b * a.C + c, o);
#pragma unroll
  for (int j = 0; j < W - 1; ++j) *reinterpret_cast<typename V::raw*>(st + (size_t)j * a.C) = r[j + 1];
}

// Workgroup: 64 channel vectors x 4 consecutive runs (a wave each) of one
// sequence.  Its sums go to partial row blockIdx.x / column blocks: W planes of
// C columns for dw, one for db.
template <typename T, int W, int VE, int ACT>
__global__ __launch_bounds__(kConvThreads) void conv_bwd_kernel(const ConvArgs a) {
  typedef VecN<T, VE> V;
  constexpr int NB = 4;
  __shared__ float buf[4][W + 1][64 * VE];
  const int CV = a.C / VE, ncb = (CV + 63) / 64;
  const unsigned rb = blockIdx.x / ncb;  // partial row: sequence and group of four runs
  const int cb = blockIdx.x - rb * ncb;
  const int groups = (a.runs + 3) / 4;
  // (a wave's run is uniform: its bounds and branches are scalar)
  const int b = rb / groups, run = 4 * (int)(rb - b * groups) + __builtin_amdgcn_readfirstlane(wave_id());
  const int cv = cb * 64 + lane_id();
  const bool mine = cv < CV;
  const int c = mine ? cv * VE : 0;
  const Seq sq = seq_of(a.cu, b, a.T);
  const int t0 = run * kConvRunB;

  float dw[W][VE], db[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    db[e] = 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) dw[j][e] = 0.f;
  }
  if (mine && (run == 0 || t0 < sq.len)) {
    const int t1 = min(t0 + kConvRunB, sq.len);
    const T* x = static_cast<const T*>(a.x) + (size_t)sq.row0 * a.ldx + c;
    const T* dy = static_cast<const T*>(a.dy) + (size_t)sq.row0 * a.C + c;
    T* dx = static_cast<T*>(a.dx) + (size_t)sq.row0 * a.C + c;
    const T* s0 = static_cast<const T*>(a.state0) + (size_t)b * (W - 1) * a.C + c;
    const T* dsT = static_cast<const T*>(a.dstateT) + (size_t)b * (W - 1) * a.C + c;
    T* ds0 = static_cast<T*>(a.dstate0) + (size_t)b * (W - 1) * a.C + c;
    float w[W][VE], bias[VE], win[W][VE], dz[W][VE];
    load_taps<W, VE>(w, a.w + (size_t)c * W);
    load_bias<VE>(bias, a.bias, c);
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        win[j][e] = 0.f;
        dz[j][e] = 0.f;
      }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
      const int p = t0 - (W - 1) + j;
      if (p >= 0 || a.state0) {
        const auto r = V::load(p >= 0 ? x + (size_t)p * a.ldx : s0 + (size_t)(p + W - 1) * a.C);
#pragma unroll
        for (int e = 0; e < VE; ++e) win[j + 1][e] = V::get(r, e);
      }
    }
    // tokens t0 .. t1 + W - 2: the last W - 1 only complete the dx before them
    const int te = t1 + W - 1;
    typename V::raw nx[NB], nd[NB];  // the rows of the next batch, requested a batch ahead
    auto request = [&](int tb) {
      if (tb < sq.len && tb < te)
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const int t = min(tb + i, sq.len - 1);
          nx[i] = V::load(x + (size_t)t * a.ldx);
          nd[i] = V::load(dy + (size_t)t * a.C);
        }
    };
    request(t0);
    for (int tb = t0; tb < te; tb += NB) {
      typename V::raw rx[NB], rd[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        rx[i] = nx[i];
        rd[i] = nd[i];
      }
      request(tb + NB);
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int t = tb + i;
        if (t >= te) break;
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            win[j][e] = win[j + 1][e];
            dz[j][e] = dz[j + 1][e];
          }
        if (t < sq.len) {
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            win[W - 1][e] = V::get(rx[i], e);
            float z = bias[e], v, d;
#pragma unroll
            for (int j = 0; j < W; ++j) z += w[j][e] * win[j][e];
            Act<T>::both(ACT, z, v, d);
            dz[W - 1][e] = V::get(rd[i], e) * d;
          }
          if (t < t1)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
              db[e] += dz[W - 1][e];
#pragma unroll
              for (int j = 0; j < W; ++j) dw[j][e] += dz[W - 1][e] * win[j][e];
            }
        } else {
#pragma unroll
          for (int e = 0; e < VE; ++e) dz[W - 1][e] = 0.f;
        }
        // dx of p = t - W + 1 is complete: dz[i] holds token p + i
        const int p = t - (W - 1);
        if (p >= t0 || (p < 0 && a.dstate0)) {
          float o[VE];
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            o[e] = 0.f;
#pragma unroll
            for (int q = 0; q < W; ++q) o[e] += w[W - 1 - q][e] * dz[q][e];
          }
          const int k = p - (sq.len - (W - 1));  // its row of the final state
          if (a.dstateT && k >= 0) {
            const auto r = V::load(dsT + (size_t)k * a.C);
#pragma unroll
            for (int e = 0; e < VE; ++e) o[e] += V::get(r, e);
          }
          V::store(p >= 0 ? dx + (size_t)p * a.C : ds0 + (size_t)(p + W - 1) * a.C, o);
        }
      }
    }
  }

  if (!a.part) return;
  const int l = lane_id(), wv = wave_id();
#pragma unroll
  for (int e = 0; e < VE; ++e) {
#pragma unroll
    for (int j = 0; j < W; ++j) buf[wv][j][l * VE + e] = dw[j][e];
    buf[wv][W][l * VE + e] = db[e];
  }
  __syncthreads();
  const int cols = min(64 * VE, a.C - cb * 64 * VE);
  for (int i = threadIdx.x; i < (W + 1) * 64 * VE; i += kConvThreads) {
    const int j = i / (64 * VE), k = i % (64 * VE);
    if (k < cols)
      a.part[((size_t)rb * (W + 1) + j) * a.C + cb * 64 * VE + k] =
          (buf[0][j][k] + buf[1][j][k]) + (buf[2][j][k] + buf[3][j][k]);
  }
}

namespace {
// 16-byte vectors; the backward holds twice as much per channel and takes four
// channels a lane.
template <typename T> constexpr int conv_ve() { return 16 / (int)sizeof(T); }
constexpr int kConvVeB = 4;

int conv_runs(int T, int len) { return T > 0 ? (T + len - 1) / len : 1; }

// The activation is a constant of the kernels: a branch on it at every element cost
// the backward 44 instead of 42 us at 12,100 packed tokens of 2048 channels.
template <typename T, int W, int ACT>
hipError_t run_conv(ConvArgs a, ConvCall call, hipStream_t st) {
  if (call == ConvCall::kBwd) {
    a.runs = conv_runs(a.T, kConvRunB);
    const long long ncb = (a.C / kConvVeB + 63) / 64;
    const long long nblk = conv_part_rows(a.B, a.T) * ncb;
    hipLaunchKernelGGL((conv_bwd_kernel<T, W, kConvVeB, ACT>), dim3((unsigned)nblk), dim3(kConvThreads), 0, st, a);
    return hipGetLastError();
  }
  constexpr int VE = conv_ve<T>();
  const long long cv = a.C / VE;
  if (call == ConvCall::kStep) {
    const long long nblk = (a.B * cv + kConvThreads - 1) / kConvThreads;
    hipLaunchKernelGGL((conv_step_kernel<T, W, VE>), dim3((unsigned)nblk), dim3(kConvThreads), 0, st, a);
    return hipGetLastError();
  }
  a.runs = conv_runs(a.T, kConvRun);
  const long long nblk = ((long long)a.B * a.runs * cv + kConvThreads - 1) / kConvThreads;
  hipLaunchKernelGGL((conv_fwd_kernel<T, W, VE, ACT>), dim3((unsigned)nblk), dim3(kConvThreads), 0, st, a);
  return hipGetLastError();
}
template <typename T, int W>
hipError_t conv_act(const ConvArgs& a, ConvCall call, hipStream_t st) {
  switch (a.act) {
    case kActNone: return run_conv<T, W, kActNone>(a, call, st);
    case kActSilu: return run_conv<T, W, kActSilu>(a, call, st);
    case kActSigmoid: return run_conv<T, W, kActSigmoid>(a, call, st);
  }
  return hipErrorInvalidValue;
}
template <typename T>
hipError_t conv_dispatch(const ConvArgs& a, int W, ConvCall call, hipStream_t st) {
  switch (W) {
    case 2: return conv_act<T, 2>(a, call, st);
    case 3: return conv_act<T, 3>(a, call, st);
    case 4: return conv_act<T, 4>(a, call, st);
  }
  return hipErrorInvalidValue;
}
}  // namespace

long long conv_part_rows(int B, int T) { return (long long)B * ((conv_runs(T, kConvRunB) + 3) / 4); }
// Thread indices, and the threads of a launch, are 32 bits wide.
bool conv_supported(int B, int T, int C, int W) {
  if (W < 2 || W > 4 || C < 8 || C % 8 || C > (1 << 24)) return false;
  const long long runs = conv_runs(T, kConvRun), ncb = (C / kConvVeB + 63) / 64;
  return (long long)B * runs * (C / 4) < (1ll << 31) - kConvThreads &&
         conv_part_rows(B, T) * ncb < (1ll << 32) / kConvThreads;
}

hipError_t launch_conv(const ConvArgs& a, int W, ConvCall call, bool is_bf16, hipStream_t st) {
  return is_bf16 ? conv_dispatch<bf16_t>(a, W, call, st) : conv_dispatch<float>(a, W, call, st);
}

// ----------------------------------------------------------------------------
// Column sums of a [rows, cols] matrix of partial sums, in a fixed order: 16
// columns per workgroup, 64 threads sharing a column's rows, eight loads in flight
// each (few rows and columns: latency is all there is).
namespace {
constexpr int kSumCols = 16, kSumRows = 64;
}
__global__ __launch_bounds__(kSumCols * kSumRows) void colsum_kernel(const ColsumArgs a) {
  __shared__ float buf[kSumRows][kSumCols + 1];
  const int cl = threadIdx.x % kSumCols, rl = threadIdx.x / kSumCols;
  const int col = (int)(blockIdx.y * gridDim.x + blockIdx.x) * kSumCols + cl;
  constexpr int U = 8;
  float s[U] = {};
  if (col < a.cols) {
    const float* p = a.part + col;
    for (long long r = rl; r < a.rows; r += U * kSumRows) {
      float x[U];
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const long long rq = r + q * kSumRows;
        x[q] = p[(size_t)(rq < a.rows ? rq : r) * a.cols];
      }
#pragma unroll
      for (int q = 0; q < U; ++q) s[q] += r + q * kSumRows < a.rows ? x[q] : 0.f;
    }
  }
  buf[rl][cl] = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
  __syncthreads();
  if (rl == 0 && col < a.cols) {
    float t = 0.f;
#pragma unroll
    for (int q = 0; q < kSumRows; ++q) t += buf[q][cl];
    if (col >= a.first) {
      if (a.out1) a.out1[col - a.first] = t;
    } else if (a.taps) {
      a.out0[(size_t)(col % a.C) * a.taps + col / a.C] = t;  // plane j, channel c -> [c][j]
    } else {
      a.out0[col] = t;
    }
  }
}

hipError_t launch_colsum(const ColsumArgs& a, hipStream_t st) {
  // (2^24 channels of four taps and a bias are 5 2^20 workgroups of 1024: more threads than one
  // dimension of a launch counts)
  const unsigned n = (unsigned)((a.cols + kSumCols - 1) / kSumCols), gx = n < (1u << 20) ? n : 1u << 20;
  hipLaunchKernelGGL(colsum_kernel, dim3(gx, (n + gx - 1) / gx), dim3(kSumCols * kSumRows), 0, st, a);
  return hipGetLastError();
}

}  // namespace ccq
