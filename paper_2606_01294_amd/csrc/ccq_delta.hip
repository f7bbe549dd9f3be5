// ccq_delta.hip -- the gated delta rule without the query contraction: the
// state pass of its chunked form for bf16 io, and the recurrent form.
//
// The chunked form is that of ccq_gdn.hip (transforms Tm, state pass, outputs),
// read with the caller's queries; value head h reads query/key head h / (HV / HK).
// Its backward is that of ccq_gdn_bwd.hip (of a few tokens, ccq_delta_short.hip).
#include <type_traits>

#include "ccq_device.h"
#include "ccq_kernels.h"
#include "ccq_plain.h"

namespace ccq {

// ----------------------------------------------------------------------------
// State pass (bf16 io), for each chunk
//
//   R = diag(beta) (V - diag(e^gamma) K S_r^T),  U = Tm R,
//   S_{r+1} = e^{gamma_C} S_r + U^T diag(e^{gamma_C - gamma}) K.
//
// K and V are exact in bf16.  S, R, Tm and U enter the products as a bf16 head
// and a bf16 tail (17 bits together; tail times tail is left out), so S_T is within
// 4e-6 of the exact state's norm, where one bf16 operand a product leaves 3e-3: a
// state that is handed on, to the next segment of a document or to the recurrent
// form, carries next to nothing of the chunked form.  S_r and U are rounded to bf16
// once, on store, for the kernels that form outputs and gradients.
//
// What bounds the pass is the chain of chunks (B HV dv / 16 value tiles of 16
// columns of S^T, a chunk after the other).  NH waves carry a tile, each DK / NH of
// its key features in accumulators, and do nothing else: splitting the features
// shortens a chunk (its products and the splitting of S into heads and tails), at
// the price of one exchange of the partial sums of K S^T through LDS.
//
// Four more waves of the workgroup stream the operands into LDS (global_load_lds,
// no registers): two take the keys of every other chunk, two chunks ahead, into a
// ring of three slots, two the transform, the values and the coefficients (X), one
// chunk ahead, into two.  A loader has one chunk in flight at most, so it waits for
// all of its loads and counts none.
//
// 1.3B forward (B = 4, T = 4096, H = 8, dk = dv = 256; features over two waves): 180 to
// 183 us (three runs of 40 launches, the least 165), 5700 cycles a chunk: 1300 of them
// products, 3300 of LDS traffic (334 KB a chunk and compute unit: K rows and transposed,
// Tm twice, the exchange), the rest the latency of the chain K S -> sum -> R -> Tm R ->
// update.  One wave a tile, in turn with it: 240 to 244 us (two tiles a workgroup), 258
// to 263 (four).  Tried without gain: a deeper key ring, loads without vector
// arithmetic, splitting S behind the update.  (Operands of one bf16 each: 100 us.)
template <int DK, int NPR, int NH>
struct DeltaTile {
  static constexpr int C = kChunk, NLW = 4, BVS = 16 * NPR, NC = NPR * NH;  // NC consumer waves
  static constexpr int KB = C * DK * 2, TB = C * C * 2, VB = C * BVS * 2, FB = 4 * C * 4;
  static constexpr int XB = 2 * TB + VB + FB, SB = NH > 1 ? NC * 4 * 64 * 16 : 0;
  static constexpr int KO = 0, XO = 3 * KB, SO = XO + 2 * XB, LDS = SO + SB;
  static constexpr int NK = KB / 1024, NT = TB / 1024, NV = VB / 1024;  // 1 KB loads
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

template <int DK, int NPR, int NH>
__global__ __launch_bounds__(64 * (NPR * NH + 4 < 8 ? 8 : NPR * NH + 4)) void delta_state_kernel(const GdnArgs a) {
  typedef bf16_t T;
  typedef __attribute__((address_space(3))) void lds_void;
  typedef DeltaTile<DK, NPR, NH> L;
  constexpr int C = kChunk, BVS = L::BVS, RB = DK * 2;
  constexpr int DKH = DK / NH, NKH = DKH / 32, NCT = DKH / 16;  // a wave's features: blocks of 32, tiles
  static_assert(NKH >= 1, "feature split");
  static_assert(L::LDS <= 160 * 1024, "LDS");
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

  if (w >= L::NC) {
    // ---- loaders: rows past the end of the sequence read the last row (finite
    // data; the chunk transform zeroes their contribution) ----
#define CCQ_LDS(src, dst) __builtin_amdgcn_global_load_lds((const void*)(src), (lds_void*)(dst), 16, 0, 0)
    const int lw = w - L::NC;
    const bool keys = lw < 2;  // waves 0, 1: keys of chunks 0, 2, .. and 1, 3, ..; 2, 3: X
    const int first = lw & 1;
    constexpr int CPK = DK / 8, CPV = BVS / 8;  // 16-byte pieces per row
    // A load covers R rows; its address is a uniform base and one of a few per-lane
    // offsets formed once (the permutation repeats every 16 rows), so issuing it
    // costs no vector arithmetic.  Rows past the end read the last row.
    if (keys) {
      constexpr int R = 64 / CPK, NP = 16 / R;
      const char* const kg = static_cast<const char*>(a.k) + 2 * seq_off(sq, 0, kh.h, kh.H, DK);
      const size_t pitch = (size_t)kh.H * RB;
      uint32_t lane[NP];
#pragma unroll
      for (int p = 0; p < NP; ++p)
        lane[p] = (l / CPK) * (uint32_t)pitch + 16 * ((l % CPK) ^ dswz<DK>(p * R + l / CPK));
      auto issue = [&](int ci) {
        char* sb = smem + L::KO + (ci % 3) * L::KB;
        const char* kc = kg + (size_t)ci * C * pitch;
        const int nrow = sq.len - ci * C;
        if (nrow >= C) {
#pragma unroll
          for (int i = 0; i < L::NK; ++i) CCQ_LDS(kc + i * R * pitch + lane[i % NP], sb + i * 1024);
        } else {
#pragma unroll 1
          for (int i = 0; i < L::NK; ++i) {
            const int row = i * R + l / CPK;
            CCQ_LDS(kc + min(row, nrow - 1) * pitch + 16 * ((l % CPK) ^ dswz<DK>(row)), sb + i * 1024);
          }
        }
      };
      if (first < NLC) issue(first);
#pragma unroll 1
      for (int ci = 0; ci < NLC; ++ci) {
        const bool mine = (ci & 1) == first;
        if (mine) wait_vm_all();
        __builtin_amdgcn_s_barrier();
        if (mine && ci + 2 < NLC) issue(ci + 2);
        if constexpr (NH > 1) __builtin_amdgcn_s_barrier();  // the consumers' exchange
      }
      return;
    }
    constexpr int R = 64 / CPV;
    const char* const vg = static_cast<const char*>(a.v) + 2 * (seq_off(sq, 0, h, a.H, a.dv) + v0);
    const size_t pitch = (size_t)a.H * a.dv * 2;
    const char* const tg = static_cast<const char*>(a.Tm) + (size_t)bh * N * L::TB;
    const char* const tl = static_cast<const char*>(a.TmLo) + (size_t)bh * N * L::TB;
    const float* const fg = a.gam + (size_t)bh * N * 5 * C;
    const uint32_t vlane = (l / CPV) * (uint32_t)pitch + 16 * (l % CPV);
    const uint32_t tlane[2] = {(uint32_t)(16 * (l & ~7) + 16 * ((l % 8) ^ tswz(l / 8))),
                               (uint32_t)(16 * (l & ~7) + 16 * ((l % 8) ^ tswz(8 + l / 8)))};
    auto issue = [&](int ci) {
      char* sb = smem + L::XO + (ci & 1) * L::XB;
      const char* vc = vg + (size_t)ci * C * pitch;
      const int nrow = sq.len - ci * C;
      if (nrow >= C) {
#pragma unroll
        for (int i = 0; i < L::NV; ++i) CCQ_LDS(vc + i * R * pitch + vlane, sb + 2 * L::TB + i * 1024);
      } else {
#pragma unroll 1
        for (int i = 0; i < L::NV; ++i)
          CCQ_LDS(vc + min(i * R + l / CPV, nrow - 1) * pitch + 16 * (l % CPV), sb + 2 * L::TB + i * 1024);
      }
      // coefficient rows 1..4: beta e^gamma, beta, e^{gamma_C - gamma}, e^{gamma_C}
      CCQ_LDS(fg + ((size_t)ci * 5 + 1) * C + 4 * l, sb + 2 * L::TB + L::VB);
#pragma unroll
      for (int i = 0; i < L::NT; ++i) {
        CCQ_LDS(tg + (size_t)ci * L::TB + i * 1024 + tlane[i % 2], sb + i * 1024);
        CCQ_LDS(tl + (size_t)ci * L::TB + i * 1024 + tlane[i % 2], sb + L::TB + i * 1024);
      }
    };
    if (first == 0 && NLC > 0) issue(0);
#pragma unroll 1
    for (int ci = 0; ci < NLC; ++ci) {
      const bool mine = (ci & 1) == first;
      if (mine) wait_vm_all();
      __builtin_amdgcn_s_barrier();
      if (!mine && ci + 1 < NLC) issue(ci + 1);
      if constexpr (NH > 1) __builtin_amdgcn_s_barrier();
    }
    return;
#undef CCQ_LDS
  }

  // ---- consumer wave: features c0 .. of value tile pr of the workgroup's slice ----
  const int pr = w / NH, hq = w % NH, c0 = hq * DKH;
  const int v = v0 + 16 * pr + c16;
  // S^T[c][v] in pair order: c = c0 + pair_feat(tc, g4) + r
  f32x4 S[NCT];
#pragma unroll
  for (int tc = 0; tc < NCT; ++tc) S[tc] = zero4();
  if (a.S0) {
    const float* s0 = a.S0 + ((size_t)bh * a.dv + v) * DK + c0 + 8 * g4;
#pragma unroll
    for (int tc = 0; tc < NCT; ++tc) S[tc] = *reinterpret_cast<const f32x4*>(s0 + pair_feat(tc, 0));
  }
  const int vt = (v0 >> 4) + pr;
  T* st_base = static_cast<T*>(a.states) + (((size_t)vt * (DK / 32) + hq * NKH) * 16 + c16) * 32 + 8 * g4;
  T* u_base = static_cast<T*>(a.U) + ((size_t)vt * 2 * 16 + c16) * 32 + 8 * g4;
  typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
  auto ldf = [](const char* p) {
    Frag<T> f;
    f.v = *reinterpret_cast<const bf16x8*>(p);
    return f;
  };
  auto tr = [](const char* p) { return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p); };
  // The permutation of K touches the low bits of the piece index only (four, or
  // three at dk = 64), so block m of 32 features (counted from the wave's first, M
  // = c0 / 32 + m) lies 256 (M / 4) bytes on from block M % 4.  krow: row c16, piece
  // 4 M + g4 (row operands); kcol: transposing reads, rows 4 g4 + j / 4 (j = c16),
  // piece 4 M + j % 4 (+ 8 bytes for odd tiles)
  constexpr int NQ = NKH < 4 ? NKH : 4;
  int krow[NQ], kcol[NQ];
  {
    const int rr = 4 * g4 + (c16 >> 2);
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int M = c0 / 32 + q;  // (NKH < 4: the wave's blocks lie within one group of four)
      krow[q] = c16 * RB + (M >> 2) * 256 + 16 * ((4 * (M & 3) + g4) ^ dswz<DK>(c16));
      kcol[q] = rr * RB + (M >> 2) * 256 + 16 * ((4 * (M & 3) + (c16 & 3)) ^ dswz<DK>(rr));
    }
  }
  const int trow = c16 * (C * 2) + 16 * (g4 ^ tswz(c16));  // Tm row c16, columns 8 g4 ..; 32 on: ^ 64
  const int vrow = (4 * g4 + (c16 >> 2)) * (2 * BVS) + 32 * pr + 8 * (c16 & 3);
  f32x4* const sX = reinterpret_cast<f32x4*>(smem + L::SO);

  // S as operands: head and tail, renewed tile by tile behind the update's products
  Frag<T> sh[NKH], sl[NKH];
#pragma unroll
  for (int m = 0; m < NKH; ++m) split_pair(S[2 * m], S[2 * m + 1], sh[m], sl[m]);
  int until = 0;  // chunks until the next stored state
#pragma unroll 1
  for (int ci = 0; ci < NLC; ++ci) {
    const char* kb = smem + L::KO + (ci % 3) * L::KB;
    const char* th = smem + L::XO + (ci & 1) * L::XB;
    const char* tl = th + L::TB;
    const char* vb = tl + L::TB;
    const float* Fb = reinterpret_cast<const float*>(vb + L::VB);
    lds_barrier();  // this chunk's operands have landed, the slots of the one before are free
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
    read_k(0);
    f32x4 R[4], bv[4], bg[4];
    Frag<T> tmh[4][2], tml[4][2];
    // Tm (rows stored in acc_pos order; the second half of rows 0..31 is zero),
    // beta V and beta e^gamma, requested among the products
    auto read_tm = [&](int I) {
      tmh[I][0] = ldf(th + trow + 16 * I * (C * 2));
      tml[I][0] = ldf(tl + trow + 16 * I * (C * 2));
      if (I >= 2) {
        tmh[I][1] = ldf(th + (trow ^ 64) + 16 * I * (C * 2));
        tml[I][1] = ldf(tl + (trow ^ 64) + 16 * I * (C * 2));
      }
    };
    auto read_v = [&](int J) {
      const bf16x4 vv = tr(vb + vrow + 16 * J * 2 * BVS);
      const f32x4 bj = *reinterpret_cast<const f32x4*>(Fb + C + 16 * J + 4 * g4);
      bg[J] = *reinterpret_cast<const f32x4*>(Fb + 16 * J + 4 * g4);
#pragma unroll
      for (int r = 0; r < 4; ++r) bv[J][r] = bj[r] * f32(vv[r]);
    };
    const float eC = Fb[3 * C];
    f32x4 x[4][2];
    // a tile's sums, one tile behind its products: the partial ones to the exchange,
    // or (one wave a value tile) R itself
    auto finish = [&](int J) {
      R[J] = x[J][0] + x[J][1];
      if constexpr (NH > 1) {
        sX[(w * 4 + J) * 64 + l] = R[J];
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) R[J][r] = bv[J][r] - bg[J][r] * R[J][r];
      }
    };
#pragma unroll
    for (int J = 0; J < 4; ++J) {
      x[J][0] = zero4();
      x[J][1] = zero4();
#pragma unroll
      for (int gb = 0; gb < NGB; ++gb) {
        const int step = J * NGB + gb;
        if (step + 1 < 4 * NGB) read_k(step + 1);
        if (gb == NGB - 1) {
          read_v(J);
          if (NH > 1 && J > 0) read_tm(J - 1);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int m = 0; m < GB; ++m) {
          mma(x[J][0], kf[step & 1][m], sh[gb * GB + m]);
          mma(x[J][1], kf[step & 1][m], sl[gb * GB + m]);
        }
      }
#pragma unroll
      for (int t = J * NCT / 4; t < (J + 1) * NCT / 4; ++t) S[t] *= eC;
      if (J > 0) finish(J - 1);
    }
    finish(3);
    if constexpr (NH > 1) {
      read_tm(3);
      lds_barrier();
      // the tile's partial sums in a fixed order: its waves hold the same bits
#pragma unroll
      for (int J = 0; J < 4; ++J) {
        f32x4 sum = sX[(pr * NH * 4 + J) * 64 + l];
#pragma unroll
        for (int hh = 1; hh < NH; ++hh) sum += sX[((pr * NH + hh) * 4 + J) * 64 + l];
#pragma unroll
        for (int r = 0; r < 4; ++r) R[J][r] = bv[J][r] - bg[J][r] * sum[r];
      }
    } else {
#pragma unroll
      for (int I = 0; I < 4; ++I) read_tm(I);
    }
    Frag<T> rh[2], rl[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) split_pair(R[2 * q], R[2 * q + 1], rh[q], rl[q]);
    // K^T of TB feature tiles at a time, for the update
    constexpr int TB = NCT < 4 ? NCT : 4;
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
    // S_r (every sstride-th chunk) and U^T, fragment-native
    if (until == 0) {
      T* st_out = st_base + ((size_t)bh * N + ci) * a.dv * DK;
#pragma unroll
      for (int m = 0; m < NKH; ++m) store_frag(st_out + 16 * 32 * m, sh[m]);
      until = a.sstride;
    }
    --until;
    if (hq == 0) {
      T* u_out = u_base + ((size_t)bh * N + ci) * a.dv * C;
      store_frag(u_out, uf[0]);
      store_frag(u_out + 16 * 32, uf[1]);
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
      if (tb4 > 0)
#pragma unroll
        for (int m = TB / 2 * (tb4 - 1); m < TB / 2 * tb4; ++m) split_pair(S[2 * m], S[2 * m + 1], sh[m], sl[m]);
    }
#pragma unroll
    for (int m = NKH - TB / 2; m < NKH; ++m) split_pair(S[2 * m], S[2 * m + 1], sh[m], sl[m]);
  }

  if (a.ST) {
    float* st = a.ST + ((size_t)bh * a.dv + v) * DK + c0 + 8 * g4;
#pragma unroll
    for (int tc = 0; tc < NCT; ++tc) *reinterpret_cast<f32x4*>(st + pair_feat(tc, 0)) = S[tc];
  }
}

// ----------------------------------------------------------------------------
// Reverse scan of D = dL/dS_{r+1} (bf16 io), last chunk to first, with dO the
// upstream gradient and s the read scale (see ccq_gdn_bwd.hip):
//
//   dU = diag(e^{gamma_C - gamma}) K D^T + s P^T dO,   dR = Tm^T dU,   dV = diag(beta) dR,
//   D <- e^{gamma_C} D + Q^T (s diag(e^gamma) dO) - K^T diag(beta e^gamma) dR.
//
// dV is stored, and D (as it enters the chunk) and dR for the chunk-parallel gradients.
// Bound, as the state pass, by the chain of chunks and laid out like it: NH
// consumer waves a value tile of 16 columns of D^T, the features of a tile split
// over them (one exchange of the partial dU), four waves that only stream.  K and
// X (P^T, Tm^T, dO, coefficients) come one chunk ahead into two slots each; Q, which
// only the end of a chunk reads, into one: its loads go out when the chunk begins, as
// those of X, those of K behind the exchange (a wave with that many loads to issue
// would hold the barrier there: 127 against 105 us at 512 tiles of dk = 128 with all
// three behind it, 109 with all before), and a barrier stands before Q's products.
// dR and dV leave through LDS and two loaders: stored by the consumers themselves,
// two bytes a lane and row, dR held them up.  Operands are bf16 (Tm^T its head alone, s e^gamma dO
// rounded once), D and every sum fp32 (D and dR are rounded as operands and on store): the
// gradients are 2.5e-3 to 3.5e-3 from the exact ones where storing them in bf16 alone leaves
// 1.7e-3; tails as further operands would lengthen the chain, which is what the scan takes.
// 1.3B training step (B = 4, T = 4096, H = 8, dk = dv = 256): 335 us in the form of
// gdn_dstate_kernel, which stages through registers, 235 to 240 in this one.
template <int DK, int NPR, int NH>
struct DeltaBackTile {
  static constexpr int C = kChunk, NLW = 4, BVS = 16 * NPR, NC = NPR * NH;
  static constexpr int KB = C * DK * 2, TB = C * C * 2, VB = C * BVS * 2, FB = 5 * C * 4;
  static constexpr int XB = 2 * TB + VB + FB, SB = NH > 1 ? NC * 4 * 64 * 16 : 0;
  static constexpr int QO = 2 * KB, XO = QO + KB, SO = XO + 2 * XB, RO = SO + SB;
  // dR and dV on their way out: over P^T, which the exchange releases, or apart
  static constexpr int LDS = RO + (NH > 1 ? 0 : 2 * VB);
  static_assert(2 * VB <= TB || NH == 1, "dR and dV over P^T");
  static constexpr int NK = KB / 1024, NT = TB / 1024, NV = VB / 1024;  // 1 KB loads
};

template <int DK, int NPR, int NH>
__global__ __launch_bounds__(64 * (NPR * NH + 4 < 8 ? 8 : NPR * NH + 4)) void delta_dstate_kernel(const GdnDstateArgs a) {
  typedef bf16_t T;
  typedef __attribute__((address_space(3))) void lds_void;
  typedef DeltaBackTile<DK, NPR, NH> L;
  constexpr int C = kChunk, BVS = L::BVS, RB = DK * 2;
  constexpr int DKH = DK / NH, NKH = DKH / 32, NCT = DKH / 16;
  static_assert(NKH >= 1 && L::LDS <= 160 * 1024, "feature split, LDS");
  __shared__ __align__(1024) char smem[L::LDS];

  const int nvt = a.dv / BVS;
  const int N = (a.T + C - 1) / C;
  const int lb = xcd_logical_block(blockIdx.x, gridDim.x);
  const int hm = lb / nvt;
  const int bh = (hm % a.B) * a.H + hm / a.B;
  const int b = bh / a.H, h = bh % a.H;
  const KeyHead kh = key_head(a.HK, a.H, h);
  const Seq sq = seq_of(a.cu, b, a.T), sp = padded_rows(sq, b, a.T);
  const int NLC = (sq.len + C - 1) / C;
  const int l = lane_id(), g4 = l >> 4, c16 = l & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int v0 = (lb % nvt) * BVS;

  if (w >= L::NC) {
    // ---- loaders: wave 0 the keys, 1 and 2 half of the queries each, 3 X.  Rows
    // past the end read the last row: P^T, Tm^T and the coefficients are zero there.  A wave waits for all its loads.
#define CCQ_LDS(src, dst) __builtin_amdgcn_global_load_lds((const void*)(src), (lds_void*)(dst), 16, 0, 0)
    const int lw = w - L::NC;
    constexpr int CPK = DK / 8, CPV = BVS / 8, R = 64 / CPK, NP = 16 / R, RV = 64 / CPV;
    const size_t pitch = (size_t)kh.H * RB, vpitch = (size_t)a.H * a.dv * 2;
    uint32_t lane[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p)
      lane[p] = (l / CPK) * (uint32_t)pitch + 16 * ((l % CPK) ^ dswz<DK>(p * R + l / CPK));
    // loads i0 .. i1 of the [C, DK] tile of chunk ci at base
    auto rows = [&](const char* base, int ci, char* dst, int i0, auto n) {
      const char* src = base + (size_t)ci * C * pitch;
      const int nrow = sq.len - ci * C;
      if (nrow >= C) {
#pragma unroll
        for (int i = 0; i < decltype(n)::value; ++i)
          CCQ_LDS(src + (size_t)(i0 + i) * R * pitch + lane[i % NP], dst + (i0 + i) * 1024);
      } else {
#pragma unroll 1
        for (int i = i0; i < i0 + decltype(n)::value; ++i) {
          const int row = i * R + l / CPK;
          CCQ_LDS(src + min(row, nrow - 1) * pitch + 16 * ((l % CPK) ^ dswz<DK>(row)), dst + i * 1024);
        }
      }
    };
    const size_t head = 2 * seq_off(sq, 0, kh.h, kh.H, DK);
    if (lw == 0) {
      const char* const kg = static_cast<const char*>(a.k) + head;
      auto issue = [&](int ci) { rows(kg, ci, smem + (ci & 1) * L::KB, 0, std::integral_constant<int, L::NK>()); };
      if (NLC > 0) issue(NLC - 1);
#pragma unroll 1
      for (int ci = NLC - 1; ci >= 0; --ci) {
        wait_vm_all();
        __builtin_amdgcn_s_barrier();
        if constexpr (NH > 1) __builtin_amdgcn_s_barrier();
        if (ci > 0) issue(ci - 1);
        __builtin_amdgcn_s_barrier();
      }
    } else if (lw < 3) {
      static_assert(L::NK / 2 % NP == 0, "half a tile begins a period of the permutation");
      const char* const qg = static_cast<const char*>(a.qc) + head;
#pragma unroll 1
      for (int ci = NLC - 1; ci >= 0; --ci) {
        __builtin_amdgcn_s_barrier();
        rows(qg, ci, smem + L::QO, (lw - 1) * (L::NK / 2), std::integral_constant<int, L::NK / 2>());
        if constexpr (NH > 1) __builtin_amdgcn_s_barrier();
        wait_vm_all();
        __builtin_amdgcn_s_barrier();
        // the chunk's dR (to the workspace) and dV (to the caller), whole rows of the slice
        const int nrow = sq.len - ci * C;
        char* const out = lw == 1 ? static_cast<char*>(a.dR) + 2 * (seq_off(sp, ci * C, h, a.H, a.dv) + v0)
                                  : static_cast<char*>(a.dv_out) + 2 * (seq_off(sq, ci * C, h, a.H, a.dv) + v0);
        const char* const from = smem + (NH > 1 ? L::XO + (ci & 1) * L::XB : L::RO) + (lw - 1) * L::VB + 16 * l;
#pragma unroll
        for (int i = 0; i < L::NV; ++i) {
          const int row = i * RV + l / CPV;
          const bf16x8 x = *reinterpret_cast<const bf16x8*>(from + i * 1024);
          if (row < nrow) *reinterpret_cast<bf16x8*>(out + row * vpitch + 16 * (l % CPV)) = x;
        }
      }
    } else {
      const char* const og = static_cast<const char*>(a.dO) + 2 * (seq_off(sq, 0, h, a.H, a.dv) + v0);
      const char* const pg = static_cast<const char*>(a.PT) + (size_t)bh * N * L::TB;
      const char* const tg = static_cast<const char*>(a.TmT) + (size_t)bh * N * L::TB;
      const float* const fg = a.gam + (size_t)bh * N * 5 * C;
      const uint32_t vlane = (l / CPV) * (uint32_t)vpitch + 16 * (l % CPV);
      const uint32_t tlane[2] = {(uint32_t)(16 * (l & ~7) + 16 * ((l % 8) ^ tswz(l / 8))),
                                 (uint32_t)(16 * (l & ~7) + 16 * ((l % 8) ^ tswz(8 + l / 8)))};
      auto issue = [&](int ci) {
        char* sb = smem + L::XO + (ci & 1) * L::XB;
        const char* oc = og + (size_t)ci * C * vpitch;
        const int nrow = sq.len - ci * C;
        CCQ_LDS(fg + (size_t)ci * 5 * C + 4 * l, sb + 2 * L::TB + L::VB);
        if (l < 16) CCQ_LDS(fg + ((size_t)ci * 5 + 4) * C + 4 * l, sb + 2 * L::TB + L::VB + 1024);
        if (nrow >= C) {
#pragma unroll
          for (int i = 0; i < L::NV; ++i) CCQ_LDS(oc + i * RV * vpitch + vlane, sb + 2 * L::TB + i * 1024);
        } else {
#pragma unroll 1
          for (int i = 0; i < L::NV; ++i)
            CCQ_LDS(oc + min(i * RV + l / CPV, nrow - 1) * vpitch + 16 * (l % CPV), sb + 2 * L::TB + i * 1024);
        }
#pragma unroll
        for (int i = 0; i < L::NT; ++i) {
          CCQ_LDS(pg + (size_t)ci * L::TB + i * 1024 + tlane[i % 2], sb + i * 1024);
          CCQ_LDS(tg + (size_t)ci * L::TB + i * 1024 + tlane[i % 2], sb + L::TB + i * 1024);
        }
      };
      if (NLC > 0) issue(NLC - 1);
#pragma unroll 1
      for (int ci = NLC - 1; ci >= 0; --ci) {
        wait_vm_all();
        // s e^gamma, zero past the end, over gamma
        float* const F = reinterpret_cast<float*>(smem + L::XO + (ci & 1) * L::XB + 2 * L::TB + L::VB);
        F[l] = l < sq.len - ci * C ? a.scale * __expf(F[l]) : 0.f;
        lds_barrier();
        if (ci > 0) issue(ci - 1);
        if constexpr (NH > 1) __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_s_barrier();
      }
    }
    return;
#undef CCQ_LDS
  }

  // ---- consumer wave: features c0 .. of value tile pr of the workgroup's slice ----
  const int pr = w / NH, hq = w % NH, c0 = hq * DKH;
  f32x4 D[NCT];  // D^T[c][v] in pair order: c = c0 + pair_feat(tc, g4) + r
#pragma unroll
  for (int tc = 0; tc < NCT; ++tc) D[tc] = zero4();
  typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
  auto ldf = [](const char* p) {
    Frag<T> f;
    f.v = *reinterpret_cast<const bf16x8*>(p);
    return f;
  };
  auto tr = [](const char* p) { return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p); };
  auto pair = [](bf16x4 lo, bf16x4 hi) {
    Frag<T> f;
    f.v = bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return f;
  };
  // offsets into the K and Q tiles, as in the state pass
  constexpr int NQ = NKH < 4 ? NKH : 4;
  int krow[NQ], kcol[NQ];
  {
    const int rr = 4 * g4 + (c16 >> 2);
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int M = c0 / 32 + q;
      krow[q] = c16 * RB + (M >> 2) * 256 + 16 * ((4 * (M & 3) + g4) ^ dswz<DK>(c16));
      kcol[q] = rr * RB + (M >> 2) * 256 + 16 * ((4 * (M & 3) + (c16 & 3)) ^ dswz<DK>(rr));
    }
  }
  const int trow = c16 * (C * 2) + 16 * (g4 ^ tswz(c16));  // Tm^T row c16, slots 8 g4 ..; 32 on: ^ 64
  // P^T row c16 in accumulator order: columns 4 g4 .. and 16 + 4 g4 .. (32 on: ^ 64)
  const int prow = c16 * (C * 2) + 8 * (g4 & 1) + 16 * ((g4 >> 1) ^ tswz(c16)), prow2 = prow ^ 32;
  const int vrow = (4 * g4 + (c16 >> 2)) * (2 * BVS) + 32 * pr + 8 * (c16 & 3);
  f32x4* const sX = reinterpret_cast<f32x4*>(smem + L::SO);
  T* const dst = static_cast<T*>(a.dstates) + ((((size_t)bh * N * (a.dv / 16) + (v0 >> 4) + pr) * (DK / 32) + hq * NKH) * 16 + c16) * 32 + 8 * g4;
  const int rrow = (4 * g4 + 2 * (c16 & 1)) * 2 * BVS + 32 * pr + 2 * (c16 & ~1);

#pragma unroll 1
  for (int ci = NLC - 1; ci >= 0; --ci) {
    const char* kb = smem + (ci & 1) * L::KB;
    const char* qb = smem + L::QO;
    const char* pb = smem + L::XO + (ci & 1) * L::XB;
    const char* tb = pb + L::TB;
    const char* ob = tb + L::TB;
    const float* Fb = reinterpret_cast<const float*>(ob + L::VB);
    Frag<T> df[NKH];
#pragma unroll
    for (int m = 0; m < NKH; ++m) df[m] = acc_pair_frag<T>(D[2 * m], D[2 * m + 1]);
    lds_barrier();  // K and X have landed; Q's slot and the others' second ones are free
    // partial dU: K D^T over the wave's features, and P^T dO for its share of the
    // token tiles; LDS reads run a group ahead of their products
    constexpr int GB = NKH < 4 ? NKH : 4, NGB = NKH / GB;
    Frag<T> kf[2][GB];
    auto read_k = [&](int step) {
      const int J = step / NGB, m0 = (step % NGB) * GB;
#pragma unroll
      for (int m = 0; m < GB; ++m)
        kf[step & 1][m] = ldf(kb + krow[(m0 + m) & 3] + ((m0 + m) >> 2) * 256 + 16 * J * RB);
    };
    read_k(0);
    Frag<T> of[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) of[q] = pair(tr(ob + vrow + 32 * q * 2 * BVS), tr(ob + vrow + (32 * q + 16) * 2 * BVS));
    {  // D, as it enters the chunk, fragment-native
      T* out = dst + (size_t)ci * a.dv * DK;
#pragma unroll
      for (int m = 0; m < NKH; ++m) store_frag(out + 16 * 32 * m, df[m]);
    }
    const float eC = Fb[4 * C];
    f32x4 dU[4];
    Frag<T> tt[4][2];
#pragma unroll
    for (int J = 0; J < 4; ++J) {
      f32x4 x[2] = {zero4(), zero4()};
      Frag<T> pf[2];
      const bool mine = J % NH == hq;
#pragma unroll
      for (int gb = 0; gb < NGB; ++gb) {
        const int step = J * NGB + gb;
        if (step + 1 < 4 * NGB) read_k(step + 1);
        if (gb == NGB - 1) {
          if (mine) {  // (P^T is zero left of the diagonal tiles)
            auto half = [&](int q) {
              return pair(*reinterpret_cast<const bf16x4*>(pb + (prow ^ (64 * q)) + 16 * J * (C * 2)),
                          *reinterpret_cast<const bf16x4*>(pb + (prow2 ^ (64 * q)) + 16 * J * (C * 2)));
            };
            if (J < 2) pf[0] = half(0);
            pf[1] = half(1);
          }
          if (J < 2) tt[J][0] = ldf(tb + trow + 16 * J * (C * 2));
          tt[J][1] = ldf(tb + (trow ^ 64) + 16 * J * (C * 2));
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int m = 0; m < GB; ++m) mma(x[m & 1], kf[step & 1][m], df[gb * GB + m]);
      }
      const f32x4 cf = *reinterpret_cast<const f32x4*>(Fb + 3 * C + 16 * J + 4 * g4);
      dU[J] = cf * (x[0] + x[1]);
      if (mine) {
        f32x4 y = zero4();
        if (J < 2) mma(y, pf[0], of[0]);
        mma(y, pf[1], of[1]);
        dU[J] += a.scale * y;
      }
      if constexpr (NH > 1) sX[(w * 4 + J) * 64 + l] = dU[J];
    }
    // s e^gamma dO, and the first K^T tiles of the update
    Frag<T> og[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      f32x4 lo = *reinterpret_cast<const f32x4*>(Fb + 32 * q + 4 * g4);
      f32x4 hi = *reinterpret_cast<const f32x4*>(Fb + 32 * q + 16 + 4 * g4);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        lo[r] *= frag_elem(of[q], r);
        hi[r] *= frag_elem(of[q], 4 + r);
      }
      og[q] = acc_pair_frag<T>(lo, hi);
    }
    constexpr int TB = NCT < 4 ? NCT : 4;
    Frag<T> tf[2][TB][2];
    auto read_t = [&](const char* base, int tc0, Frag<T>(&f)[TB][2]) {
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        const int tc = tc0 + t, m = tc >> 1;
        const char* p = base + kcol[m & 3] + (m >> 2) * 256 + 8 * (tc & 1);
#pragma unroll
        for (int kq = 0; kq < 2; ++kq) f[t][kq] = pair(tr(p + 32 * kq * RB), tr(p + (32 * kq + 16) * RB));
      }
    };
    read_t(kb, 0, tf[0]);
    if constexpr (NH > 1) {
      lds_barrier();
      // the tile's partial sums in a fixed order: its waves hold the same bits
#pragma unroll
      for (int J = 0; J < 4; ++J) {
        f32x4 sum = sX[(pr * NH * 4 + J) * 64 + l];
#pragma unroll
        for (int hh = 1; hh < NH; ++hh) sum += sX[((pr * NH + hh) * 4 + J) * 64 + l];
        dU[J] = sum;
      }
    }
    f32x4 bg[4];
#pragma unroll
    for (int I = 0; I < 4; ++I) bg[I] = *reinterpret_cast<const f32x4*>(Fb + C + 16 * I + 4 * g4);
    const Frag<T> uf0 = acc_pair_frag<T>(dU[0], dU[1]), uf1 = acc_pair_frag<T>(dU[2], dU[3]);
    f32x4 dR[4];
#pragma unroll
    for (int I = 0; I < 4; ++I) {
      dR[I] = zero4();
      mma(dR[I], tt[I][1], uf1);
    }
#pragma unroll
    for (int I = 0; I < 2; ++I) mma(dR[I], tt[I][0], uf0);
#pragma unroll
    for (int t = 0; t < NCT; ++t) D[t] *= eC;
    f32x4 dRb[4];
#pragma unroll
    for (int I = 0; I < 4; ++I) dRb[I] = dR[I] * -bg[I];
    const Frag<T> rf[2] = {acc_pair_frag<T>(dRb[0], dRb[1]), acc_pair_frag<T>(dRb[2], dRb[3])};
#pragma unroll
    for (int tb4 = 0; tb4 < NCT / TB; ++tb4) {
      if (tb4 + 1 < NCT / TB) read_t(kb, TB * (tb4 + 1), tf[(tb4 + 1) & 1]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kq = 0; kq < 2; ++kq)
#pragma unroll
        for (int t = 0; t < TB; ++t) mma(D[TB * tb4 + t], tf[tb4 & 1][t][kq], rf[kq]);
    }
    // dR and dV to LDS, token-major: a lane holds four tokens of one column;
    // neighbours swap two of them, so that each writes two tokens of two columns
    char* const ro = smem + (NH > 1 ? L::XO + (ci & 1) * L::XB : L::RO) + rrow;
    auto out = [&](const f32x4& x, char* to_) {
      typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));
      const bool odd = c16 & 1;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float keep = odd ? x[2 + r] : x[r], got = lane_swap(odd ? x[r] : x[2 + r]);
        *reinterpret_cast<bf16x2*>(to_ + r * 2 * BVS) = bf16x2{to<T>(odd ? got : keep), to<T>(odd ? keep : got)};
      }
    };
#pragma unroll
    for (int I = 0; I < 4; ++I)
      if (I % NH == hq) {
        out(dR[I], ro + 16 * I * 2 * BVS);
        out(dR[I] * *reinterpret_cast<const f32x4*>(Fb + 2 * C + 16 * I + 4 * g4), ro + L::VB + 16 * I * 2 * BVS);
      }
    lds_barrier();  // Q has landed, dR and dV are in LDS
    read_t(qb, 0, tf[0]);
#pragma unroll
    for (int tb4 = 0; tb4 < NCT / TB; ++tb4) {
      if (tb4 + 1 < NCT / TB) read_t(qb, TB * (tb4 + 1), tf[(tb4 + 1) & 1]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kq = 0; kq < 2; ++kq)
#pragma unroll
        for (int t = 0; t < TB; ++t) mma(D[TB * tb4 + t], tf[tb4 & 1][t][kq], og[kq]);
    }
  }
}

// ----------------------------------------------------------------------------
// Recurrent form on the fp32 state, in place, for one or a few tokens:
//   u = beta (v - alpha S k),  o = scale (alpha S q + (k . q) u),  S <- alpha S + u k^T.
// Every row of S goes through the tokens on its own, so a row is read once and
// written once whatever T is; 16 lanes hold a row (each 16-byte pieces j, j + 16,
// ..), a workgroup kStepRows rows of one head.  Bound by HBM (S in and out): 64
// sequences of the 1.3B layer's 8 heads, 270 MB of state traffic, 42 us.
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
// over the value heads of a query/key head, in order.  Bound by HBM (12,100 packed
// tokens, 8 value heads on 4, dk = 128: 22 us for 112 MB).
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
template <int DK, int NPR, int NH>
hipError_t run_delta_state(const GdnArgs& a, hipStream_t st) {
  typedef DeltaTile<DK, NPR, NH> L;
  const int nblk = a.B * a.H * (a.dv / (16 * NPR));
  if (nblk == 0) return hipSuccess;
  hipLaunchKernelGGL((delta_state_kernel<DK, NPR, NH>), dim3(nblk), dim3(64 * (L::NC + L::NLW)), 0, st, a);
  return hipGetLastError();
}
// Value tiles a workgroup and waves a tile, by the number of tiles (state pass
// alone, 32 chunks): a compute unit to every tile while there are enough, the
// features then split where that pays; from there on more tiles a workgroup, so
// that all of them run at once.
//   dk = 256:  128 tiles  69 us at 1 x 4 waves, 83 at 2 x 2;   512: 84 at 2 x 2, 133 at 1 x 4;
//             1024        153 at 2 x 2, 249 at 1 x 4
//   dk = 128:  128        57 at 1 x 4, 61 at 2 x 1, 63 at 4 x 1;  512: 63 at 2 x 1, 66 at 2 x 2;
//             1024        70 at 4 x 1, 116 at 2 x 1, 190 at 8 x 1
//   dk = 64:    64        42 at 2 x 1, 45 at 1 x 2;  512: 44 at 2 x 1, 48 at 4 x 1;
//             2048        49 at 8 x 1, 59 at 4 x 1, 93 at 2 x 1
template <int DK>
hipError_t run_delta_state_dk(const GdnArgs& a, hipStream_t st) {
  const long long tiles = (long long)a.B * a.H * (a.dv / 16);
  if constexpr (DK == 64) {
    if (tiles > 1024 && a.dv % 128 == 0) return run_delta_state<DK, 8, 1>(a, st);
    if (tiles > 512) return run_delta_state<DK, 4, 1>(a, st);
    return run_delta_state<DK, 2, 1>(a, st);
  } else {
    if (tiles <= 256) return run_delta_state<DK, 1, 4>(a, st);
    if constexpr (DK == 256) return run_delta_state<DK, 2, 2>(a, st);
    else if (tiles > 512) return run_delta_state<DK, 4, 1>(a, st);
    else return run_delta_state<DK, 2, 1>(a, st);
  }
}
template <int DK, int NPR, int NH>
hipError_t run_delta_dstate(const GdnDstateArgs& a, hipStream_t st) {
  typedef DeltaBackTile<DK, NPR, NH> L;
  const int nblk = a.B * a.H * (a.dv / (16 * NPR));
  if (nblk == 0) return hipSuccess;
  hipLaunchKernelGGL((delta_dstate_kernel<DK, NPR, NH>), dim3(nblk), dim3(64 * (L::NC + L::NLW)), 0, st, a);
  return hipGetLastError();
}
// Value tiles a workgroup and waves a tile, as for the state pass (the scan alone,
// 32 chunks):
//   dk = 256:  128 tiles  65 us at 1 x 4 waves, 86 at 2 x 2;  512: 103 at 2 x 2, 145 at 1 x 4
//   dk = 128:  128        55 at 1 x 4, 60 at 2 x 1;   512: 76 at 2 x 2 and at 2 x 1, 91 at 4 x 1;
//             1024       112 at 4 x 1, 154 at 2 x 2, 161 at 8 x 1
//   dk = 64:    64        53 at 2 x 1, 52 at 1 x 2;   512: 72 at 2 x 1, 79 at 4 x 1
// and, with 16 chunks, 2048 tiles: 96 at 8 x 1, 112 at 4 x 1 (dk = 128), 74 and 91 (dk = 64).
template <int DK>
hipError_t run_delta_dstate_dk(const GdnDstateArgs& a, hipStream_t st) {
  const long long tiles = (long long)a.B * a.H * (a.dv / 16);
  if constexpr (DK == 256) {
    return tiles <= 256 ? run_delta_dstate<DK, 1, 4>(a, st) : run_delta_dstate<DK, 2, 2>(a, st);
  } else {
    if (tiles > 1024 && a.dv % 128 == 0) return run_delta_dstate<DK, 8, 1>(a, st);
    if (tiles > 512) return run_delta_dstate<DK, 4, 1>(a, st);
    if constexpr (DK == 64) return run_delta_dstate<DK, 2, 1>(a, st);
    else return tiles <= 256 ? run_delta_dstate<DK, 1, 4>(a, st) : run_delta_dstate<DK, 2, 2>(a, st);
  }
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

hipError_t launch_delta_dstate(const GdnDstateArgs& a, hipStream_t st) {
  switch (a.dk) {
    case 64: return run_delta_dstate_dk<64>(a, st);
    case 128: return run_delta_dstate_dk<128>(a, st);
    case 256: return run_delta_dstate_dk<256>(a, st);
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
