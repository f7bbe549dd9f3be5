// ccq_layer_api.cpp -- the part of the C ABI (include/ccq.h) around the query
// contraction: the plain gated delta rule, the short convolution, the head norm.
// Every check runs before the first launch, as in ccq_api.cpp.
#include <cmath>

#include "ccq.h"
#include "ccq_api_util.h"
#include "ccq_kernels.h"

using namespace ccq_api;

namespace {

bool present(const void* p) { return p && aligned(p); }
bool optional_ok(const void* p) { return !p || aligned(p); }
bool offsets_ok(const int32_t* cu) { return cu && (reinterpret_cast<uintptr_t>(cu) & 3u) == 0; }
bool overlap(const void* p, size_t n, const void* q, size_t m) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return p && q && a < b + m && b < a + n;
}

// Whether n bytes at p meet the first `width` bytes of one of `rows` rows, `pitch` bytes apart, at x.
bool meets_rows(const void* p, size_t n, const void* x, size_t rows, size_t pitch, size_t width) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(x);
  if (!p || !x || n == 0 || rows == 0) return false;
  const size_t i = a < b + width ? 0 : (a - b - width) / pitch + 1;  // the first row that ends behind p
  return i < rows && b + i * pitch < a + n;
}

// ---- delta rule ------------------------------------------------------------
bool delta_rows_ok(const ccq_delta_shape* s) { return (long long)s->HV * (s->dk > s->dv ? s->dk : s->dv) <= (1LL << 24); }
ccq_status check_delta(const ccq_delta_shape* s, bool bwd) {
  if (!s) return CCQ_ERR_INVALID_ARG;
  if (s->B < 0 || s->T < 0 || s->HK < 0 || s->HV < 0 || !dtype_ok(s->io_dtype)) return CCQ_ERR_INVALID_ARG;
  if (s->HV > 0 && (s->HK == 0 || s->HV % s->HK != 0)) return CCQ_ERR_INVALID_ARG;
  const bool bf = s->io_dtype == CCQ_BF16;
  if (!ccq::gdn_supported(s->dk, s->dv, bf)) return CCQ_ERR_UNSUPPORTED;
  if (bwd && !ccq::bwd_supported(s->dk, s->dv, bf, true)) return CCQ_ERR_UNSUPPORTED;
  // 64-bit token offsets; a launch's threads (up to 512 a chunk, 256 a tile of 16 value
  // channels at dk = 256, 128 below) and the offsets within a chunk are 32 bits wide
  const long long bh = (long long)s->B * s->HV;
  if (bh * ((s->T + 63LL) / 64) >= (1LL << 23) || !delta_rows_ok(s)) return CCQ_ERR_UNSUPPORTED;
  if (bh * s->dv >= (s->dk == 256 ? 1LL << 28 : 1LL << 29)) return CCQ_ERR_UNSUPPORTED;
  if (bh * s->T * (s->dk > s->dv ? s->dk : s->dv) > (1LL << 40)) return CCQ_ERR_UNSUPPORTED;
  return CCQ_OK;
}

struct DeltaLayout {
  size_t states = 0, Tm = 0, TmLo = 0, gam = 0, gamLo = 0, U = 0;  // forward
  size_t PT = 0, TmT = 0, dstates = 0, dR = 0, dq = 0, dk = 0;  // training step
  size_t hist = 0, part = 0, gpart = 0;                         // the same, a few tokens
  size_t total = 0;
};
DeltaLayout delta_layout(const ccq_delta_shape* s, bool bwd) {
  DeltaLayout L;
  const size_t ntok = (size_t)s->B * s->T * s->HV;
  const size_t nchunk = (size_t)s->B * s->HV * (((size_t)s->T + 63) / 64);
  const size_t e = esize(s->io_dtype);
  auto take = [&](size_t bytes) { const size_t o = L.total; L.total += align_up(bytes); return o; };
  L.states = take(nchunk * s->dv * s->dk * e);
  L.Tm = take(nchunk * 64 * 64 * e);
  if (s->io_dtype == CCQ_BF16) L.TmLo = take(nchunk * 64 * 64 * e);
  L.gam = take(nchunk * 5 * 64 * sizeof(float));
  L.gamLo = take(nchunk * 64 * sizeof(float));
  L.U = take(nchunk * 64 * s->dv * e);
  if (bwd && ccq::delta_short(s->B, s->T, s->HV, s->io_dtype == CCQ_BF16)) {
    L.hist = take(ccq::delta_short_hist(s->B, s->T, s->HV, s->dk, s->dv) * sizeof(float));
    L.part = take(ccq::delta_short_part(s->B, s->T, s->HV, s->dk, s->dv) * sizeof(float));
    L.gpart = take(ccq::delta_short_gpart(s->B, s->T, s->HV, s->dv) * sizeof(float));
  } else if (bwd) {
    L.PT = take(nchunk * 64 * 64 * e);
    L.TmT = take(nchunk * 64 * 64 * e);
    L.dstates = take(nchunk * s->dv * s->dk * e);
    L.dR = take(ntok * s->dv * e);
    if (s->HK != s->HV) {
      L.dq = take(ntok * s->dk * sizeof(float));
      L.dk = take(ntok * s->dk * sizeof(float));
    }
  }
  return L;
}

struct DeltaGrads {
  const void* dO;
  void *dq, *dk, *dv, *dla, *dbeta;
};

ccq_status run_delta(const ccq_delta_shape* s, const int32_t* cu, bool packed, const void* q, const void* k,
                     const void* v, const float* la, const float* beta, const float* S0, void* o, float* ST,
                     const DeltaGrads* g, void* workspace, size_t ws_bytes, void* stream) {
  ccq_status rc = check_delta(s, g != nullptr);
  if (rc != CCQ_OK) return rc;
  if (packed && s->B > 65535) return CCQ_ERR_UNSUPPORTED;
  if (s->B == 0 || s->HV == 0) return CCQ_OK;
  if (packed && !offsets_ok(cu)) return CCQ_ERR_INVALID_ARG;
  if (!optional_ok(S0) || !optional_ok(ST) || !optional_ok(workspace)) return CCQ_ERR_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const size_t state_bytes = (size_t)s->B * s->HV * s->dv * s->dk * sizeof(float);
  if (ST && ST != S0 && overlap(S0, state_bytes, ST, state_bytes)) return CCQ_ERR_INVALID_ARG;
  if (s->T == 0) {
    if (ST && ST != S0 && ccq::launch_copy_or_zero(ST, S0, state_bytes / sizeof(float), st) != hipSuccess)
      return CCQ_ERR_HIP;
    return CCQ_OK;
  }
  const void* req[] = {q, k, v, la, beta};
  for (const void* p : req)
    if (!present(p)) return CCQ_ERR_INVALID_ARG;
  if (g) {
    const void* grads[] = {g->dO, g->dq, g->dk, g->dv, g->dla, g->dbeta};
    for (const void* p : grads)
      if (!present(p)) return CCQ_ERR_INVALID_ARG;
  }
  if (g ? !optional_ok(o) : !present(o)) return CCQ_ERR_INVALID_ARG;
  const DeltaLayout L = delta_layout(s, g != nullptr);
  if (!workspace || ws_bytes < L.total) return CCQ_ERR_WORKSPACE;

  char* ws = static_cast<char*>(workspace);
  const bool bf = s->io_dtype == CCQ_BF16;
  const int B = s->B, T = s->T, H = s->HV;
  float* gam = reinterpret_cast<float*>(ws + L.gam);
  float* gamLo = reinterpret_cast<float*>(ws + L.gamLo);
  trace_begin_call();
  // a few tokens: the gradients token by token, the chunked form where o or ST is wanted
  const bool few = g && ccq::delta_short(B, T, H, bf);
  if (few) {
    float* const f[] = {reinterpret_cast<float*>(ws + L.hist), reinterpret_cast<float*>(ws + L.part),
                        reinterpret_cast<float*>(ws + L.gpart)};
    ccq::DeltaShortArgs da{q, k, v, g->dO, la, beta, S0, f[0], f[1], f[2], g->dq, g->dk, g->dv, g->dla, g->dbeta,
                           B, T, s->HK, H, s->dk, s->dv, s->scale, cu};
    if (traced(st, [&] { return ccq::launch_delta_short(da, st); }) != hipSuccess) return CCQ_ERR_HIP;
    if (traced(st, [&] { return ccq::launch_delta_short_sum(da, st); }) != hipSuccess) return CCQ_ERR_HIP;
    if (!o && !ST) return CCQ_OK;
    g = nullptr;
  }
  // chunk transforms and decay coefficients, then the chain of chunk states
  ccq::TriArgs ta{k, la, beta, ws + L.Tm, gam, B, T, H, s->dk, s->dv};
  ta.cu = cu;
  ta.HK = s->HK;
  ta.TmLo = bf ? ws + L.TmLo : nullptr;
  ta.gamLo = gamLo;
  if (traced(st, [&] { return ccq::launch_gdn_tri(ta, bf, st); }) != hipSuccess) return CCQ_ERR_HIP;
  const int group = ccq::gdn_out_group(B, H, T, s->dk, s->dv, bf);
  ccq::GdnArgs sa{k, v, beta, ws + L.Tm, gam, S0, ST, ws + L.states, ws + L.U, B, T, H, s->dk, s->dv};
  sa.sstride = g ? 1 : group;  // the backward reads every S_r, the outputs one per group
  sa.cu = cu;
  sa.HK = s->HK;
  sa.TmLo = ta.TmLo;
  if (traced(st, [&] { return bf ? ccq::launch_delta_state(sa, st) : ccq::launch_gdn_state(sa, false, st); }) !=
      hipSuccess)
    return CCQ_ERR_HIP;
  if (o) {
    ccq::GdnOutArgs oa{q, k, gam, ws + L.states, ws + L.U, o, B, T, H, s->dk, s->dv, s->scale};
    oa.group = group;
    oa.cu = cu;
    oa.HK = s->HK;
    oa.gamLo = gamLo;
    if (traced(st, [&] { return ccq::launch_gdn_out(oa, bf, st); }) != hipSuccess) return CCQ_ERR_HIP;
  }
  if (!g) return CCQ_OK;
  // backward: P^T and Tm^T, the reverse scan of the state's adjoint, chunk gradients
  ccq::GdnPrepArgs pa{q, k, gam, ws + L.Tm, ws + L.PT, ws + L.TmT, B, T, H, s->dk, s->dv};
  pa.cu = cu;
  pa.HK = s->HK;
  pa.gamLo = gamLo;
  if (traced(st, [&] { return ccq::launch_gdn_bwd_prep(pa, bf, st); }) != hipSuccess) return CCQ_ERR_HIP;
  ccq::GdnDstateArgs da{q, k, g->dO, gam, ws + L.PT, ws + L.TmT, ws + L.dstates, ws + L.dR, B, T, H, s->dk, s->dv,
                        s->scale};
  da.cu = cu;
  da.HK = s->HK;
  da.dv_out = g->dv;
  if (traced(st, [&] { return bf ? ccq::launch_delta_dstate(da, st) : ccq::launch_gdn_dstate(da, false, st); }) !=
      hipSuccess)
    return CCQ_ERR_HIP;
  ccq::GdnBwdArgs ba{};
  ba.qc = q;
  ba.k = k;
  ba.v = v;
  ba.dO = g->dO;
  ba.gam = gam;
  ba.states = ws + L.states;
  ba.U = ws + L.U;
  ba.dstates = ws + L.dstates;
  ba.dR = ws + L.dR;
  ba.dqc = reinterpret_cast<float*>(ws + L.dq);
  ba.dk_bb = reinterpret_cast<float*>(ws + L.dk);
  ba.dqc_io = g->dq;
  ba.dk_io = g->dk;
  ba.dv_out = g->dv;
  ba.dla_io = g->dla;
  ba.dbeta_io = g->dbeta;
  ba.B = B;
  ba.T = T;
  ba.H = H;
  ba.dk = s->dk;
  ba.dv = s->dv;
  ba.scale = s->scale;
  ba.cu = cu;
  ba.HK = s->HK;
  ba.gamLo = gamLo;
  if (traced(st, [&] { return ccq::launch_gdn_bwd_chunk(ba, bf, st); }) != hipSuccess) return CCQ_ERR_HIP;
  if (s->HK != s->HV) {
    ccq::HeadSumArgs ha{ba.dqc, ba.dk_bb, g->dq, g->dk, B, T, s->HK, H, s->dk};
    ha.cu = cu;
    if (traced(st, [&] { return ccq::launch_head_sum(ha, bf, st); }) != hipSuccess) return CCQ_ERR_HIP;
  }
  return CCQ_OK;
}

// ---- convolution -----------------------------------------------------------
bool act_ok(ccq_act a) { return a == CCQ_ACT_NONE || a == CCQ_ACT_SILU || a == CCQ_ACT_SIGMOID; }
bool pitch_ok(int64_t ld, int64_t least, ccq_dtype t) { return ld >= least && ld <= (1LL << 40) && ld * (int64_t)esize(t) % 16 == 0; }

ccq_status check_conv(const ccq_conv_shape* s) {
  if (!s) return CCQ_ERR_INVALID_ARG;
  if (s->B < 0 || s->T < 0 || s->C < 0 || !dtype_ok(s->io_dtype) || !act_ok(s->act)) return CCQ_ERR_INVALID_ARG;
  if (!ccq::conv_supported(s->B, s->T, s->C, s->W)) return CCQ_ERR_UNSUPPORTED;
  if (!pitch_ok(s->ldx, s->C, s->io_dtype)) return CCQ_ERR_INVALID_ARG;
  return CCQ_OK;
}
size_t conv_ws(const ccq_conv_shape* s) {
  return align_up((size_t)ccq::conv_part_rows(s->B, s->T) * (s->W + 1) * s->C * sizeof(float));
}

ccq_status conv_forward(const ccq_conv_shape* s, const int32_t* cu, bool packed, const void* x, const float* w,
                        const float* bias, const void* state0, void* y, void* stateT, void* stream) {
  ccq_status rc = check_conv(s);
  if (rc != CCQ_OK) return rc;
  if (s->B == 0) return CCQ_OK;
  if (packed && !offsets_ok(cu)) return CCQ_ERR_INVALID_ARG;
  if (!optional_ok(bias) || !optional_ok(state0) || !optional_ok(stateT)) return CCQ_ERR_INVALID_ARG;
  const size_t sb = (size_t)s->B * (s->W - 1) * s->C * esize(s->io_dtype);
  if (overlap(state0, sb, stateT, sb)) return CCQ_ERR_INVALID_ARG;
  if (!present(w) || (s->T > 0 && (!present(x) || !present(y)))) return CCQ_ERR_INVALID_ARG;
  // runs of tokens read the inputs ahead of their first one (rows of a packed batch are not known here)
  const size_t e = esize(s->io_dtype), rows = (size_t)s->B * s->T, yb = packed ? 0 : rows * s->C * e;
  if (overlap(y, yb, state0, sb) || overlap(y, yb, stateT, sb)) return CCQ_ERR_INVALID_ARG;
  if (!packed && (meets_rows(y, yb, x, rows, s->ldx * e, s->C * e) || meets_rows(stateT, sb, x, rows, s->ldx * e, s->C * e)))
    return CCQ_ERR_INVALID_ARG;
  if (s->T == 0 && !stateT) return CCQ_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  ccq::ConvArgs a{};
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.state0 = state0;
  a.y = y;
  a.stateT = stateT;
  a.B = s->B;
  a.T = s->T;
  a.C = s->C;
  a.act = s->act;
  a.ldx = s->ldx;
  a.cu = cu;
  trace_begin_call();
  if (traced(st, [&] { return ccq::launch_conv(a, s->W, ccq::ConvCall::kFwd, s->io_dtype == CCQ_BF16, st); }) !=
      hipSuccess)
    return CCQ_ERR_HIP;
  return CCQ_OK;
}

ccq_status conv_backward(const ccq_conv_shape* s, const int32_t* cu, bool packed, const void* x, const float* w,
                         const float* bias, const void* state0, const void* dy, const void* dstateT, void* dx,
                         float* dw, float* dbias, void* dstate0, void* workspace, size_t ws_bytes, void* stream) {
  ccq_status rc = check_conv(s);
  if (rc != CCQ_OK) return rc;
  const void* opt[] = {bias, state0, dstateT, dbias, dstate0, workspace};
  for (const void* p : opt)
    if (!optional_ok(p)) return CCQ_ERR_INVALID_ARG;
  if (!present(dw) || (bias != nullptr) != (dbias != nullptr)) return CCQ_ERR_INVALID_ARG;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (s->B == 0) {  // sums over nothing
    if (ccq::launch_copy_or_zero(dw, nullptr, (size_t)s->C * s->W, st) != hipSuccess) return CCQ_ERR_HIP;
    if (dbias && ccq::launch_copy_or_zero(dbias, nullptr, s->C, st) != hipSuccess) return CCQ_ERR_HIP;
    return CCQ_OK;
  }
  if (packed && !offsets_ok(cu)) return CCQ_ERR_INVALID_ARG;
  if (!present(w) || (s->T > 0 && (!present(x) || !present(dy) || !present(dx)))) return CCQ_ERR_INVALID_ARG;
  if (!workspace || ws_bytes < conv_ws(s)) return CCQ_ERR_WORKSPACE;
  ccq::ConvArgs a{};
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.state0 = state0;
  a.dy = dy;
  a.dstateT = dstateT;
  a.dx = dx;
  a.dstate0 = dstate0;
  a.part = static_cast<float*>(workspace);
  a.B = s->B;
  a.T = s->T;
  a.C = s->C;
  a.act = s->act;
  a.ldx = s->ldx;
  a.cu = cu;
  trace_begin_call();
  if (traced(st, [&] { return ccq::launch_conv(a, s->W, ccq::ConvCall::kBwd, s->io_dtype == CCQ_BF16, st); }) !=
      hipSuccess)
    return CCQ_ERR_HIP;
  // partial rows hold W planes of dw and one of db; without a bias only dw is summed
  ccq::ColsumArgs c{a.part, ccq::conv_part_rows(s->B, s->T), (s->W + 1) * s->C, s->W * s->C, dw, dbias, s->W, s->C};
  if (traced(st, [&] { return ccq::launch_colsum(c, st); }) != hipSuccess) return CCQ_ERR_HIP;
  return CCQ_OK;
}

// ---- norm ------------------------------------------------------------------
ccq_status check_norm(const ccq_norm_shape* s) {
  if (!s) return CCQ_ERR_INVALID_ARG;
  if (s->rows < 0 || s->G < 0 || s->D < 0 || !dtype_ok(s->io_dtype) || !act_ok(s->act)) return CCQ_ERR_INVALID_ARG;
  if (s->kind != CCQ_NORM_GROUP && s->kind != CCQ_NORM_RMS && s->kind != CCQ_NORM_L2) return CCQ_ERR_INVALID_ARG;
  if (s->shared != 0 && s->shared != 1) return CCQ_ERR_INVALID_ARG;
  if (!(s->eps >= 0.f) || std::isinf(s->eps)) return CCQ_ERR_INVALID_ARG;
  if (!ccq::norm_supported(s->D) || (long long)s->G * s->D > (1LL << 24)) return CCQ_ERR_UNSUPPORTED;
  if (s->rows > (1LL << 40) / ((long long)s->D * (s->G > 0 ? s->G : 1))) return CCQ_ERR_UNSUPPORTED;
  if (!pitch_ok(s->ldx, (int64_t)s->G * s->D, s->io_dtype)) return CCQ_ERR_INVALID_ARG;
  return CCQ_OK;
}
ccq::NormArgs norm_args(const ccq_norm_shape* s, const void* x, const float* w, const float* bias, const void* gate) {
  ccq::NormArgs a{};
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.gate = gate;
  a.rows = s->rows;
  a.ldx = s->ldx;
  a.ldg = s->ldg;
  a.G = s->G;
  a.D = s->D;
  a.kind = s->kind;
  a.act = s->act;
  a.shared = s->shared;
  a.eps = s->eps;
  return a;
}
long long norm_cols(const ccq_norm_shape* s) { return (long long)(s->shared ? 1 : s->G) * s->D; }

}  // namespace

extern "C" {

size_t ccq_delta_workspace_size(const ccq_delta_shape* s, int with_bwd) {
  return check_delta(s, with_bwd != 0) == CCQ_OK ? delta_layout(s, with_bwd != 0).total : 0;
}

ccq_status ccq_delta_fwd(const ccq_delta_shape* s, const void* q, const void* k, const void* v, const float* logalpha,
                         const float* beta, const float* S0, void* o, float* ST, void* workspace, size_t ws_bytes,
                         void* stream) {
  return run_delta(s, nullptr, false, q, k, v, logalpha, beta, S0, o, ST, nullptr, workspace, ws_bytes, stream);
}

ccq_status ccq_delta_fwd_varlen(const ccq_delta_shape* s, const int32_t* cu_seqlens, const void* q, const void* k,
                                const void* v, const float* logalpha, const float* beta, const float* S0, void* o,
                                float* ST, void* workspace, size_t ws_bytes, void* stream) {
  return run_delta(s, cu_seqlens, true, q, k, v, logalpha, beta, S0, o, ST, nullptr, workspace, ws_bytes, stream);
}

ccq_status ccq_delta_fwd_bwd(const ccq_delta_shape* s, const void* q, const void* k, const void* v,
                             const float* logalpha, const float* beta, const float* S0, const void* dO, void* o,
                             float* ST, void* dq, void* dk, void* dv, void* dlogalpha, void* dbeta, void* workspace,
                             size_t ws_bytes, void* stream) {
  const DeltaGrads g{dO, dq, dk, dv, dlogalpha, dbeta};
  return run_delta(s, nullptr, false, q, k, v, logalpha, beta, S0, o, ST, &g, workspace, ws_bytes, stream);
}

ccq_status ccq_delta_fwd_bwd_varlen(const ccq_delta_shape* s, const int32_t* cu_seqlens, const void* q, const void* k,
                                    const void* v, const float* logalpha, const float* beta, const float* S0,
                                    const void* dO, void* o, float* ST, void* dq, void* dk, void* dv, void* dlogalpha,
                                    void* dbeta, void* workspace, size_t ws_bytes, void* stream) {
  const DeltaGrads g{dO, dq, dk, dv, dlogalpha, dbeta};
  return run_delta(s, cu_seqlens, true, q, k, v, logalpha, beta, S0, o, ST, &g, workspace, ws_bytes, stream);
}

ccq_status ccq_delta_step(const ccq_delta_shape* s, const void* q, const void* k, const void* v, const float* logalpha,
                          const float* beta, float* S, void* o, void* stream) {
  if (!s) return CCQ_ERR_INVALID_ARG;
  if (s->B < 0 || s->T < 0 || s->HK < 0 || s->HV < 0 || !dtype_ok(s->io_dtype)) return CCQ_ERR_INVALID_ARG;
  if (s->HV > 0 && (s->HK == 0 || s->HV % s->HK != 0)) return CCQ_ERR_INVALID_ARG;
  if (!ccq::decode_supported(s->dk, s->dv)) return CCQ_ERR_UNSUPPORTED;
  // 16 threads a row of the state, and a launch's threads are 32 bits wide
  if ((long long)s->B * s->HV * s->dv >= (1LL << 28) || !delta_rows_ok(s)) return CCQ_ERR_UNSUPPORTED;
  if (s->B == 0 || s->HV == 0 || s->T == 0) return CCQ_OK;
  const void* req[] = {q, k, v, logalpha, beta, S, o};
  for (const void* p : req)
    if (!present(p)) return CCQ_ERR_INVALID_ARG;
  const ccq::DeltaStepArgs a{q, k, v, logalpha, beta, S, o, s->B, s->T, s->HK, s->HV, s->dk, s->dv, s->scale};
  hipStream_t st = static_cast<hipStream_t>(stream);
  trace_begin_call();
  if (traced(st, [&] { return ccq::launch_delta_step(a, s->io_dtype == CCQ_BF16, st); }) != hipSuccess)
    return CCQ_ERR_HIP;
  return CCQ_OK;
}

ccq_status ccq_conv_fwd(const ccq_conv_shape* s, const void* x, const float* w, const float* bias, const void* state0,
                        void* y, void* stateT, void* stream) {
  return conv_forward(s, nullptr, false, x, w, bias, state0, y, stateT, stream);
}

ccq_status ccq_conv_fwd_varlen(const ccq_conv_shape* s, const int32_t* cu_seqlens, const void* x, const float* w,
                               const float* bias, const void* state0, void* y, void* stateT, void* stream) {
  return conv_forward(s, cu_seqlens, true, x, w, bias, state0, y, stateT, stream);
}

size_t ccq_conv_workspace_size(const ccq_conv_shape* s) { return check_conv(s) == CCQ_OK ? conv_ws(s) : 0; }

ccq_status ccq_conv_bwd(const ccq_conv_shape* s, const void* x, const float* w, const float* bias, const void* state0,
                        const void* dy, const void* dstateT, void* dx, float* dw, float* dbias, void* dstate0,
                        void* workspace, size_t ws_bytes, void* stream) {
  return conv_backward(s, nullptr, false, x, w, bias, state0, dy, dstateT, dx, dw, dbias, dstate0, workspace, ws_bytes,
                       stream);
}

ccq_status ccq_conv_bwd_varlen(const ccq_conv_shape* s, const int32_t* cu_seqlens, const void* x, const float* w,
                               const float* bias, const void* state0, const void* dy, const void* dstateT, void* dx,
                               float* dw, float* dbias, void* dstate0, void* workspace, size_t ws_bytes, void* stream) {
  return conv_backward(s, cu_seqlens, true, x, w, bias, state0, dy, dstateT, dx, dw, dbias, dstate0, workspace,
                       ws_bytes, stream);
}

ccq_status ccq_conv_step(const ccq_conv_shape* s, const void* x, const float* w, const float* bias, void* state, void* y,
                         void* stream) {
  ccq_status rc = check_conv(s);
  if (rc != CCQ_OK) return rc;
  if (s->T != 1) return CCQ_ERR_INVALID_ARG;
  if (s->B == 0) return CCQ_OK;
  if (!present(x) || !present(w) || !optional_ok(bias) || !present(state) || !present(y)) return CCQ_ERR_INVALID_ARG;
  ccq::ConvArgs a{};
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.y = y;
  a.stateT = state;
  a.B = s->B;
  a.T = 1;
  a.C = s->C;
  a.act = s->act;
  a.ldx = s->ldx;
  hipStream_t st = static_cast<hipStream_t>(stream);
  trace_begin_call();
  if (traced(st, [&] { return ccq::launch_conv(a, s->W, ccq::ConvCall::kStep, s->io_dtype == CCQ_BF16, st); }) !=
      hipSuccess)
    return CCQ_ERR_HIP;
  return CCQ_OK;
}

ccq_status ccq_norm_fwd(const ccq_norm_shape* s, const void* x, const float* w, const float* bias, const void* gate,
                        void* y, void* stream) {
  ccq_status rc = check_norm(s);
  if (rc != CCQ_OK) return rc;
  if (s->rows == 0 || s->G == 0) return CCQ_OK;
  if (!present(x) || !present(y) || !optional_ok(w) || !optional_ok(bias) || !optional_ok(gate)) return CCQ_ERR_INVALID_ARG;
  if ((bias && !w) || (gate && !pitch_ok(s->ldg, (int64_t)s->G * s->D, s->io_dtype))) return CCQ_ERR_INVALID_ARG;
  ccq::NormArgs a = norm_args(s, x, w, bias, gate);
  a.y = y;
  hipStream_t st = static_cast<hipStream_t>(stream);
  trace_begin_call();
  if (traced(st, [&] { return ccq::launch_norm(a, s->io_dtype == CCQ_BF16, false, st); }) != hipSuccess)
    return CCQ_ERR_HIP;
  return CCQ_OK;
}

size_t ccq_norm_workspace_size(const ccq_norm_shape* s) {
  if (check_norm(s) != CCQ_OK) return 0;
  if (s->rows == 0 || s->G == 0) return 0;
  return align_up((size_t)ccq::norm_part_rows(s->rows, s->G, s->D, s->shared) * norm_cols(s) * 2 * sizeof(float));
}

ccq_status ccq_norm_bwd(const ccq_norm_shape* s, const void* x, const float* w, const float* bias, const void* gate,
                        const void* dy, void* dx, float* dw, float* dbias, void* dgate, void* workspace,
                        size_t ws_bytes, void* stream) {
  ccq_status rc = check_norm(s);
  if (rc != CCQ_OK) return rc;
  const void* opt[] = {w, bias, gate, dw, dbias, dgate, workspace};
  for (const void* p : opt)
    if (!optional_ok(p)) return CCQ_ERR_INVALID_ARG;
  if ((bias && !w) || (w != nullptr) != (dw != nullptr) || (bias != nullptr) != (dbias != nullptr))
    return CCQ_ERR_INVALID_ARG;
  const long long cols = norm_cols(s);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (s->rows == 0 || s->G == 0) {  // sums over nothing
    if (dw && ccq::launch_copy_or_zero(dw, nullptr, cols, st) != hipSuccess) return CCQ_ERR_HIP;
    if (dbias && ccq::launch_copy_or_zero(dbias, nullptr, cols, st) != hipSuccess) return CCQ_ERR_HIP;
    return CCQ_OK;
  }
  if (!present(x) || !present(dy) || !present(dx) || (gate != nullptr) != (dgate != nullptr)) return CCQ_ERR_INVALID_ARG;
  if (gate && !pitch_ok(s->ldg, (int64_t)s->G * s->D, s->io_dtype)) return CCQ_ERR_INVALID_ARG;
  if (w && (!workspace || ws_bytes < ccq_norm_workspace_size(s))) return CCQ_ERR_WORKSPACE;
  ccq::NormArgs a = norm_args(s, x, w, bias, gate);
  a.dy = dy;
  a.dx = dx;
  a.dgate = dgate;
  a.part = w ? static_cast<float*>(workspace) : nullptr;
  trace_begin_call();
  if (traced(st, [&] { return ccq::launch_norm(a, s->io_dtype == CCQ_BF16, true, st); }) != hipSuccess)
    return CCQ_ERR_HIP;
  if (!w) return CCQ_OK;
  const ccq::ColsumArgs c{a.part, ccq::norm_part_rows(s->rows, s->G, s->D, s->shared), (int)(bias ? 2 * cols : cols),
                          (int)cols, dw, dbias, 0, 0};
  if (traced(st, [&] { return ccq::launch_colsum(c, st); }) != hipSuccess) return CCQ_ERR_HIP;
  return CCQ_OK;
}

}  // extern "C"
