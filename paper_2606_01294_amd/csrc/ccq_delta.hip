// ccq_delta.hip -- the gated delta rule without the query contraction: the
// state pass of its chunked form for bf16 io, and the recurrent form.
//
// The chunked form is that of ccq_gdn.hip (transforms Tm, state pass, outputs),
// read with the caller's queries; value head h reads query/key head h / (HV / HK).
// Its backward is that of ccq_gdn_bwd.hip.
#include "ccq_device.h"
#include "ccq_kernels.h"

namespace ccq {

// ----------------------------------------------------------------------------
// State pass (bf16 io), for each chunk
//
//   R = diag(beta) (V - diag(e^gamma) K S_r^T),  U = Tm R,
//   S_{r+1} = e^{gamma_C} S_r + U^T diag(e^{gamma_C - gamma}) K.
//
// K and V are exact in bf16.  S, R, Tm and U enter the products as a bf16 head
// and a bf16 tail (17 bits together; tail times tail is left out), so S_T comes
// out as exact as fp32 arithmetic makes it (2e-6 of its norm, where one bf16
// operand a product leaves 3e-3): a state that is handed on, to the next segment
// of a document or to the recurrent form, carries no rounding of the chunked
// form.  S_r and U are rounded to bf16 once, on store, for the kernels that form
// outputs and gradients.
//
// What bounds the pass is the chain of chunks (B HV dv / 16 value tiles, a chunk
// after the other), so one wave carries a value tile whole (16 columns of S^T,
// all key features, in accumulators) and does nothing else; four more waves of
// the workgroup stream the next chunk's operands into the other of two LDS slots
// (global_load_lds, no registers).  One barrier a chunk.
template <int DK, int NPR>
struct DeltaTile {
  static constexpr int C = kChunk, NLW = 4, BVS = 16 * NPR, NKH = DK / 32;
  static constexpr int KB = C * DK * 2, TB = C * C * 2, VB = C * BVS * 2, FB = 4 * C * 4;
  static constexpr int SB = KB + 2 * TB + VB + FB, NSLOT = 2, LDS = NSLOT * SB;
  static constexpr int NKL = KB / 1024 / NLW, NTL = TB / 1024 / NLW, NV = VB / 1024;  // 1 KB loads
};

template <int DK>
__device__ __forceinline__ int dswz(int r) {
  if constexpr (DK == 64) return tswz(r);
  else return kswz(r);
}

// x, y (two accumulator tiles) as an operand fragment's head and tail.
__device__ __forceinline__ void split_pair(const f32x4& x, const f32x4& y, Frag<bf16_t>& hi, Frag<bf16_t>& lo) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    bf16_t h, t;
    split_bf16(x[e], h, t);
    hi.v[e] = h;
    lo.v[e] = t;
    split_bf16(y[e], h, t);
    hi.v[4 + e] = h;
    lo.v[4 + e] = t;
  }
}

template <int DK, int NPR>
__global__ __launch_bounds__(64 * (NPR + 4 < 8 ? 8 : NPR + 4)) void delta_state_kernel(const GdnArgs a) {
  typedef bf16_t T;
  typedef __attribute__((address_space(3))) void lds_void;
  typedef DeltaTile<DK, NPR> L;
  constexpr int C = kChunk, BVS = L::BVS, NKH = L::NKH, NCT = DK / 16, RB = DK * 2;
  static_assert(L::LDS <= 160 * 1024 && L::NKL >= 1 && L::KB / 1024 % L::NLW == 0, "LDS and load split");
  __shared__ __align__(1024) char smem[L::LDS];

  const int nvt = a.dv / BVS;
  const int N = (a.T + C - 1) / C;
  const int lb = xcd_logical_block(blockIdx.x, gridDim.x);
  const int hm = lb / nvt;  // heads in head-major order, as gdn_state_kernel
  const int bh = (hm % a.B) * a.H + hm / a.B;
  const int b = bh / a.H, h = bh % a.H;
  const KeyHead kh = key_head(a.HK, a.H, h);
  const Seq sq = seq_of(a.cu, b, a.T);
  const int NLC = (sq.len + C - 1) / C;  // chunks walked (a packed sequence's own)
  const int l = lane_id(), g4 = l >> 4, c16 = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int v0 = (lb % nvt) * BVS;

  if (w >= NPR) {
    // ---- loaders: rows past the end of the sequence read the last row (finite
    // data; the chunk transform zeroes their contribution) ----
#define CCQ_LDS(src, dst) __builtin_amdgcn_global_load_lds((const void*)(src), (lds_void*)(dst), 16, 0, 0)
    const int lw = w - NPR;
    const char* const kg = static_cast<const char*>(a.k);
    const char* const vg = static_cast<const char*>(a.v);
    const char* const tg = static_cast<const char*>(a.Tm) + (size_t)bh * N * L::TB;
    const char* const tl = static_cast<const char*>(a.TmLo) + (size_t)bh * N * L::TB;
    const float* const fg = a.gam + (size_t)bh * N * 5 * C;
    constexpr int CPK = DK / 8, CPV = BVS / 8;  // 16-byte pieces per row
    auto issue = [&](int ci) {
      char* sb = smem + (ci % L::NSLOT) * L::SB;
      const int nrow = min(C, sq.len - ci * C);
      const char* kc = kg + seq_off(sq, ci * C, kh.h, kh.H, DK) * 2;
      const char* vc = vg + (seq_off(sq, ci * C, h, a.H, a.dv) + v0) * 2;
#pragma unroll
      for (int it = 0; it < L::NKL; ++it) {
        const int i = L::NLW * it + lw, row = i * (64 / CPK) + l / CPK;
        CCQ_LDS(kc + (size_t)min(row, nrow - 1) * (kh.H * RB) + 16 * ((l % CPK) ^ dswz<DK>(row)), sb + i * 1024);
      }
#pragma unroll
      for (int it = 0; it < L::NTL; ++it) {
        const int i = L::NLW * it + lw, row = i * 8 + l / 8;
        const size_t off = (size_t)ci * L::TB + row * (C * 2) + 16 * ((l % 8) ^ tswz(row));
        CCQ_LDS(tg + off, sb + L::KB + i * 1024);
        CCQ_LDS(tl + off, sb + L::KB + L::TB + i * 1024);
      }
#pragma unroll
      for (int i = lw; i < L::NV; i += L::NLW) {
        const int row = i * (64 / CPV) + l / CPV;
        CCQ_LDS(vc + (size_t)min(row, nrow - 1) * (a.H * a.dv * 2) + 16 * (l % CPV), sb + L::KB + 2 * L::TB + i * 1024);
      }
      // coefficient rows 1..4: beta e^gamma, beta, e^{gamma_C - gamma}, e^{gamma_C}
      if (lw == L::NLW - 1) CCQ_LDS(fg + ((size_t)ci * 5 + 1) * C + 4 * l, sb + L::KB + 2 * L::TB + L::VB);
    };
    if (NLC > 0) issue(0);
    // At the barrier of chunk ci its slot has landed and the consumers are done
    // with the other one, which chunk ci + 1 then takes: its loads have a whole
    // chunk's time.
#pragma unroll 1
    for (int ci = 0; ci < NLC; ++ci) {
      wait_vm_all();
      __builtin_amdgcn_s_barrier();
      if (ci + 1 < NLC) issue(ci + 1);
    }
    return;
#undef CCQ_LDS
  }

  // ---- consumer wave: value tile w of the workgroup's slice ----
  const int v = v0 + 16 * w + c16;
  // S^T[c][v] in pair order: c = pair_feat(tc, g4) + r
  f32x4 S[NCT];
#pragma unroll
  for (int tc = 0; tc < NCT; ++tc) S[tc] = zero4();
  if (a.S0) {
    const float* s0 = a.S0 + ((size_t)bh * a.dv + v) * DK + 8 * g4;
#pragma unroll
    for (int tc = 0; tc < NCT; ++tc) S[tc] = *reinterpret_cast<const f32x4*>(s0 + pair_feat(tc, 0));
  }
  const int vt = (v0 >> 4) + w;
  T* st_base = static_cast<T*>(a.states) + ((size_t)vt * NKH * 16 + c16) * 32 + 8 * g4;
  T* u_base = static_cast<T*>(a.U) + ((size_t)vt * 2 * 16 + c16) * 32 + 8 * g4;
  typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
  auto ldf = [](const char* p) {
    Frag<T> f;
    f.v = *reinterpret_cast<const bf16x8*>(p);
    return f;
  };
  auto tr = [](const char* p) { return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p); };
  // The permutation of K touches the low bits of the piece index only (four, or
  // three at dk = 64), so a lane's block m of 32 features lies 256 (m / 4) bytes
  // on from block m % 4.  krow: row c16, piece 4 m + g4 (row operands); kcol:
  // transposing reads, rows 4 g4 + j / 4 (j = c16), piece 4 m + j % 4 (+ 8 bytes
  // for odd tiles)
  constexpr int NQ = NKH < 4 ? NKH : 4;
  int krow[NQ], kcol[NQ];
  {
    const int rr = 4 * g4 + (c16 >> 2);
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      krow[q] = c16 * RB + 16 * ((4 * q + g4) ^ dswz<DK>(c16));
      kcol[q] = rr * RB + 16 * ((4 * q + (c16 & 3)) ^ dswz<DK>(rr));
    }
  }
  const int trow = c16 * (C * 2) + 16 * (g4 ^ tswz(c16));  // Tm row c16, columns 8 g4 ..; 32 on: ^ 64
  const int vrow = (4 * g4 + (c16 >> 2)) * (2 * BVS) + 32 * w + 8 * (c16 & 3);

  int until = 0;  // chunks until the next stored state
#pragma unroll 1
  for (int ci = 0; ci < NLC; ++ci) {
    const char* kb = smem + (ci % L::NSLOT) * L::SB;
    const char* th = kb + L::KB;
    const char* tl = th + L::TB;
    const char* vb = tl + L::TB;
    const float* Fb = reinterpret_cast<const float*>(vb + L::VB);
    Frag<T> sh[NKH], sl[NKH];
#pragma unroll
    for (int m = 0; m < NKH; ++m) split_pair(S[2 * m], S[2 * m + 1], sh[m], sl[m]);
    lds_barrier();  // this chunk's slot has landed, the other one is free
    // R = beta V - beta e^gamma K S_r^T, token tile J in accumulators.  LDS reads
    // run one group of GB feature blocks ahead of their products (the scheduling
    // barriers keep the compiler from sinking them): the wave is alone on its
    // SIMD's matrix core, so nothing else hides them.
    constexpr int GB = NKH < 4 ? NKH : 4, NGB = NKH / GB;
    Frag<T> kf[2][GB];
    auto read_k = [&](int step) {
      const int J = step / NGB, m0 = (step % NGB) * GB;
#pragma unroll
      for (int m = 0; m < GB; ++m)
        kf[step & 1][m] = ldf(kb + krow[(m0 + m) & 3] + ((m0 + m) >> 2) * 256 + 16 * J * RB);
    };
    const float eC = Fb[3 * C];
    read_k(0);
    f32x4 R[4];
    Frag<T> tmh[4][2], tml[4][2];
#pragma unroll
    for (int J = 0; J < 4; ++J) {
      const bf16x4 vv = tr(vb + vrow + 16 * J * 2 * BVS);
      const f32x4 bg = *reinterpret_cast<const f32x4*>(Fb + 16 * J + 4 * g4);
      const f32x4 bj = *reinterpret_cast<const f32x4*>(Fb + C + 16 * J + 4 * g4);
      f32x4 x[4];
#pragma unroll
      for (int g = 0; g < 4; ++g) x[g] = zero4();
#pragma unroll
      for (int gb = 0; gb < NGB; ++gb) {
        const int step = J * NGB + gb;
        if (step + 1 < 4 * NGB) {
          read_k(step + 1);
        } else {  // Tm (rows stored in acc_pos order; the second half of rows 0..31 is zero)
#pragma unroll
          for (int I = 0; I < 4; ++I) {
            tmh[I][0] = ldf(th + trow + 16 * I * (C * 2));
            tml[I][0] = ldf(tl + trow + 16 * I * (C * 2));
            if (I >= 2) {
              tmh[I][1] = ldf(th + (trow ^ 64) + 16 * I * (C * 2));
              tml[I][1] = ldf(tl + (trow ^ 64) + 16 * I * (C * 2));
            }
          }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int m = 0; m < GB; ++m) {
          mma(x[m & 1], kf[step & 1][m], sh[gb * GB + m]);
          mma(x[2 + (m & 1)], kf[step & 1][m], sl[gb * GB + m]);
        }
      }
#pragma unroll
      for (int t = 0; t < NCT / 4; ++t) S[NCT / 4 * J + t] *= eC;
      const f32x4 sum = (x[0] + x[1]) + (x[2] + x[3]);
#pragma unroll
      for (int r = 0; r < 4; ++r) R[J][r] = bj[r] * f32(vv[r]) - bg[r] * sum[r];
    }
    Frag<T> rh[2], rl[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) split_pair(R[2 * q], R[2 * q + 1], rh[q], rl[q]);
    // K^T of TB feature tiles at a time, for the update
    constexpr int TB = 4;
    Frag<T> tf[2][TB][2];
    auto read_t = [&](int tc0, Frag<T>(&f)[TB][2]) {
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        const int tc = tc0 + t, m = tc >> 1;
        const char* pk = kb + kcol[m & 3] + (m >> 2) * 256 + 8 * (tc & 1);
#pragma unroll
        for (int kq = 0; kq < 2; ++kq) {
          const bf16x4 lo = tr(pk + 32 * kq * RB), hi = tr(pk + (32 * kq + 16) * RB);
          f[t][kq].v = bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        }
      }
    };
    f32x4 dd[4];
#pragma unroll
    for (int I = 0; I < 4; ++I) dd[I] = *reinterpret_cast<const f32x4*>(Fb + 2 * C + 16 * I + 4 * g4);
    read_t(0, tf[0]);
    __builtin_amdgcn_sched_barrier(0);
    // U = Tm R
    f32x4 U[4];
#pragma unroll
    for (int I = 0; I < 4; ++I) {
      U[I] = zero4();
      mma(U[I], tml[I][0], rh[0]);
    }
#pragma unroll
    for (int I = 0; I < 4; ++I) mma(U[I], tmh[I][0], rl[0]);
#pragma unroll
    for (int I = 2; I < 4; ++I) mma(U[I], tml[I][1], rh[1]);
#pragma unroll
    for (int I = 2; I < 4; ++I) mma(U[I], tmh[I][1], rl[1]);
#pragma unroll
    for (int I = 0; I < 4; ++I) mma(U[I], tmh[I][0], rh[0]);
#pragma unroll
    for (int I = 2; I < 4; ++I) mma(U[I], tmh[I][1], rh[1]);
    Frag<T> uf[2], uh[2], ul[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      uf[q] = acc_pair_frag<T>(U[2 * q], U[2 * q + 1]);
      U[2 * q] *= dd[2 * q];
      U[2 * q + 1] *= dd[2 * q + 1];
      split_pair(U[2 * q], U[2 * q + 1], uh[q], ul[q]);
    }
    // S^T <- e^{gamma_C} S^T + K^T diag(e^{gamma_C - gamma}) U
#pragma unroll
    for (int tb4 = 0; tb4 < NCT / TB; ++tb4) {
      if (tb4 + 1 < NCT / TB) read_t(TB * (tb4 + 1), tf[(tb4 + 1) & 1]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kq = 0; kq < 2; ++kq) {
#pragma unroll
        for (int t = 0; t < TB; ++t) mma(S[TB * tb4 + t], tf[tb4 & 1][t][kq], ul[kq]);
#pragma unroll
        for (int t = 0; t < TB; ++t) mma(S[TB * tb4 + t], tf[tb4 & 1][t][kq], uh[kq]);
      }
    }
    // S_r (every sstride-th chunk) and U^T, fragment-native
    if (until == 0) {
      T* st_out = st_base + ((size_t)bh * N + ci) * a.dv * DK;
#pragma unroll
      for (int m = 0; m < NKH; ++m) store_frag(st_out + 16 * 32 * m, sh[m]);
      until = a.sstride;
    }
    --until;
    T* u_out = u_base + ((size_t)bh * N + ci) * a.dv * C;
    store_frag(u_out, uf[0]);
    store_frag(u_out + 16 * 32, uf[1]);
  }

  if (a.ST) {
    float* st = a.ST + ((size_t)bh * a.dv + v) * DK + 8 * g4;
#pragma unroll
    for (int tc = 0; tc < NCT; ++tc) *reinterpret_cast<f32x4*>(st + pair_feat(tc, 0)) = S[tc];
  }
}

// ----------------------------------------------------------------------------
// Recurrent form on the fp32 state, in place, for one or a few tokens:
//   u = beta (v - alpha S k),  o = scale (alpha S q + (k . q) u),  S <- alpha S + u k^T.
// Every row of S goes through the tokens on its own, so a row is read once and
// written once whatever T is; 16 lanes hold a row (each 16-byte pieces j, j + 16,
// ..), a workgroup kStepRows rows of one head.  Bound by HBM (S in and out).
namespace {
constexpr int kStepThreads = 256, kStepTpr = 16;
constexpr int kStepRows = kStepThreads / kStepTpr;
}  // namespace

template <typename T, int DK>
__global__ __launch_bounds__(kStepThreads) void delta_step_kernel(const DeltaStepArgs a) {
  constexpr int NV = DK / (4 * kStepTpr);
  typedef T v4 __attribute__((ext_vector_type(4)));
  const int nb = a.dv / kStepRows;
  const int bh = blockIdx.x / nb, r = (blockIdx.x % nb) * kStepRows + threadIdx.x / kStepTpr;
  const int b = bh / a.HV, h = bh % a.HV, j = threadIdx.x % kStepTpr;
  const KeyHead kh = key_head(a.HK, a.HV, h);
  float* const S = a.S + ((size_t)bh * a.dv + r) * DK + 4 * j;
  f32x4 x[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) x[i] = *reinterpret_cast<const f32x4*>(S + 64 * i);
  for (int t = 0; t < a.T; ++t) {
    const size_t tok = (size_t)b * a.T + t;
    const T* q = static_cast<const T*>(a.q) + (tok * kh.H + kh.h) * DK + 4 * j;
    const T* k = static_cast<const T*>(a.k) + (tok * kh.H + kh.h) * DK + 4 * j;
    const float vr = f32(static_cast<const T*>(a.v)[(tok * a.HV + h) * a.dv + r]);
    const float al = __expf(a.logalpha[tok * a.HV + h]), bt = a.beta[tok * a.HV + h];
    f32x4 kk[NV];
    float y = 0.f, z = 0.f, kq = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const v4 kv = *reinterpret_cast<const v4*>(k + 64 * i), qv = *reinterpret_cast<const v4*>(q + 64 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float ke = f32(kv[e]), qe = f32(qv[e]);
        kk[i][e] = ke;
        y += x[i][e] * ke;
        z += x[i][e] * qe;
        kq += ke * qe;
      }
    }
    y = group_sum<kStepTpr>(y);
    z = group_sum<kStepTpr>(z);
    kq = group_sum<kStepTpr>(kq);
    const float u = bt * (vr - al * y);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] = al * x[i][e] + u * kk[i][e];
    if (j == 0) static_cast<T*>(a.o)[(tok * a.HV + h) * a.dv + r] = to<T>(a.scale * (al * z + kq * u));
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) *reinterpret_cast<f32x4*>(S + 64 * i) = x[i];
}

// Gradients of shared query/key heads: dq and dk of every value head (fp32) summed
// over the value heads of a query/key head, in order.
template <typename T>
__global__ __launch_bounds__(256) void head_sum_kernel(const HeadSumArgs a) {
  const int per = a.HK * (a.dk / 4);  // four channels a thread
  const size_t n = (size_t)a.B * a.T * per;
  const int G = a.HV / a.HK;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
    const size_t tok = i / per;  // of the padded workspace
    const int b = (int)(tok / a.T), t = (int)(tok % a.T), rem = (int)(i % per);
    const Seq sq = seq_of(a.cu, b, a.T);
    if (t >= sq.len) continue;
    const int hk = rem / (a.dk / 4), ch = (rem % (a.dk / 4)) * 4;
    const size_t src = (tok * a.HV + (size_t)hk * G) * a.dk + ch, dst = seq_off(sq, t, hk, a.HK, a.dk) + ch;
    f32x4 q = zero4(), k = zero4();
    for (int g = 0; g < G; ++g) {
      q += *reinterpret_cast<const f32x4*>(a.dq + src + (size_t)g * a.dk);
      k += *reinterpret_cast<const f32x4*>(a.dk_in + src + (size_t)g * a.dk);
    }
    store4(static_cast<T*>(a.dq_out) + dst, q[0], q[1], q[2], q[3]);
    store4(static_cast<T*>(a.dk_out) + dst, k[0], k[1], k[2], k[3]);
  }
}

namespace {
template <int DK, int NPR>
hipError_t run_delta_state(const GdnArgs& a, hipStream_t st) {
  const int nblk = a.B * a.H * (a.dv / (16 * NPR));
  if (nblk == 0) return hipSuccess;
  hipLaunchKernelGGL((delta_state_kernel<DK, NPR>), dim3(nblk), dim3(64 * (NPR + DeltaTile<DK, NPR>::NLW)), 0, st, a);
  return hipGetLastError();
}
// One value tile per workgroup while every tile can have a compute unit of its
// own, else two, else four (where a workgroup's LDS admits them).
template <int DK>
hipError_t run_delta_state_dk(const GdnArgs& a, hipStream_t st) {
  const long long tiles = (long long)a.B * a.H * (a.dv / 16);
  if (tiles <= 256) return run_delta_state<DK, 1>(a, st);
  if (tiles <= 512) return run_delta_state<DK, 2>(a, st);
  return run_delta_state<DK, 4>(a, st);
}
template <typename T>
hipError_t step_dispatch(const DeltaStepArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long long)a.B * a.HV * (a.dv / kStepRows))), block(kStepThreads);
  switch (a.dk) {
    case 64: hipLaunchKernelGGL((delta_step_kernel<T, 64>), grid, block, 0, st, a); break;
    case 128: hipLaunchKernelGGL((delta_step_kernel<T, 128>), grid, block, 0, st, a); break;
    case 256: hipLaunchKernelGGL((delta_step_kernel<T, 256>), grid, block, 0, st, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}
}  // namespace

hipError_t launch_delta_state(const GdnArgs& a, hipStream_t st) {
  switch (a.dk) {
    case 64: return run_delta_state_dk<64>(a, st);
    case 128: return run_delta_state_dk<128>(a, st);
    case 256: return run_delta_state_dk<256>(a, st);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_delta_step(const DeltaStepArgs& a, bool is_bf16, hipStream_t st) {
  return is_bf16 ? step_dispatch<bf16_t>(a, st) : step_dispatch<float>(a, st);
}

hipError_t launch_head_sum(const HeadSumArgs& a, bool is_bf16, hipStream_t st) {
  const long long n = (long long)a.B * a.T * a.HK * (a.dk / 4);
  if (n == 0) return hipSuccess;
  const dim3 grid((unsigned)((n + 255) / 256 < 16384 ? (n + 255) / 256 : 16384));
  if (is_bf16) hipLaunchKernelGGL(head_sum_kernel<bf16_t>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(head_sum_kernel<float>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace ccq
