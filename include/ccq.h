/*
 * ccq.h -- C ABI of the MI355X (gfx950) Curvature-Conditioned Query library.
 *
 * Curvature-Conditioned Query (CCQ, arXiv 2606.01294) cleans every query of
 * a linear-attention layer before it reads the fast-weight state:
 *
 *     Sigma_t   = Cbar_t - mu_t mu_t^T,  Cbar_t = (1/t) sum_{j<=t} k_j k_j^T,
 *                                        mu_t   = (1/t) sum_{j<=t} k_j
 *                                        (Sec. 3.2, second-order expansion)
 *     q_clean_t = q_t - lambda_t Sigma_t q_t                     (Eq. clean)
 *     o_t       = scale * S_t q_clean_t                          (Eq. read)
 *
 * where S_t is the backbone state, written before it is read.  The library
 * computes this with the chunkwise form of Alg. 1 (App. B: the second-moment
 * and mean terms split into a carried inter-chunk state and an intra-chunk
 * block) for two backbones:
 *
 *   GLA             S_t = S_{t-1} diag(exp g_t) + v_t k_t^T,   g_t in R^{dk}
 *   Gated DeltaNet  S_t = alpha_t S_{t-1} (I - beta_t k_t k_t^T) + beta_t v_t k_t^T
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  * Every tensor argument is a DEVICE pointer owned by the caller, dense and
 *    row-major.  Token tensors are [B, T, H, d]; states are [B, H, ...].
 *    Pointers must be 16-byte aligned.
 *  * The library allocates and frees nothing.  Scratch comes from the caller's
 *    `workspace` of at least ccq_workspace_size() bytes (16-byte aligned).
 *  * Calls are asynchronous on `stream` (a hipStream_t; NULL = the null
 *    stream): every kernel of a call is launched on that stream, in order.
 *    The library creates no streams or events.  Arguments are validated
 *    before anything is launched; on an error nothing is launched and nothing
 *    is written.  A failed launch returns CCQ_ERR_HIP.  Nothing aborts,
 *    nothing throws, and nothing is kept between calls except the per-thread
 *    setting of the timing hook ccq_trace_events (off unless a caller sets
 *    it): concurrent calls on different workspaces are safe.
 *  * q and k are used as given (the caller applies any l2-normalisation, as
 *    Alg. 1 does before the cleaning lines).  NaN/Inf inputs propagate.
 *  * Statistics (Cbar, mu) and the backbone state are fp32 whatever io_dtype
 *    is; products run on the MFMA units with fp32 accumulation.
 */
#ifndef CCQ_H_
#define CCQ_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  CCQ_OK = 0,
  CCQ_ERR_INVALID_ARG = 1, /* NULL where a tensor is required, negative sizes, misalignment */
  CCQ_ERR_UNSUPPORTED = 2, /* a head size, chunk or dtype the library has no kernel for */
  CCQ_ERR_WORKSPACE = 3,   /* workspace NULL or smaller than ccq_workspace_size() */
  CCQ_ERR_HIP = 4          /* the HIP runtime reported an error at launch */
} ccq_status;

typedef enum { CCQ_F32 = 0, CCQ_BF16 = 1 } ccq_dtype;
typedef enum { CCQ_GLA = 0, CCQ_GDN = 1 } ccq_backbone;

typedef struct {
  int32_t B, T, H;      /* batch, tokens, heads (T may be any value >= 0) */
  int32_t dk, dv;       /* key / value head size: dv in {64,128,256,512}; dk in {64,128}
                         * (GLA, or fp32 io), {64,128,256} (bf16 Gated DeltaNet) */
  int32_t chunk;        /* chunk length C of Alg. 1; must be 64 */
  ccq_dtype io_dtype;   /* dtype of q, k, v, o (and of dq, dk, dv, dO in the backward) */
  ccq_dtype gate_dtype; /* dtype of the GLA gate g (and of dg); ignored for GDN */
  float scale;          /* o = scale * S q_clean; the paper's read uses 1.0 */
  int32_t centered;     /* 1: Sigma = Cbar - mu mu^T (the paper); 0: Sigma = Cbar (App. E ablation) */
  int32_t decay_aligned;/* 0: the paper's undecayed statistics.  1 (Gated DeltaNet forward only):
                         * the decay-aligned covariance Sigma^gamma that App. J names as future
                         * work for forgetting backbones, read as key j entering token t's
                         * statistics with the backbone's own decay prod_{s=j+1..t} alpha_s and
                         * t replaced by the decayed count W_t = alpha_t W_{t-1} + 1 (Alg. 2's
                         * running means with W_t for t); alpha = 1 gives Sigma_t.  Needs t0 = 0
                         * and no C0 / mu0 (the cache holds no W); CT, muT are then the
                         * weighted means.  Else CCQ_ERR_UNSUPPORTED (GLA, whose decay is per
                         * channel; ccq_fwd_bwd; ccq_decode). */
  int64_t t0;           /* tokens already absorbed into C0/mu0; positions are t0+1 .. t0+T */
} ccq_shape;

/* Bytes of device workspace the call needs (0 when none).  with_bwd selects
 * the training entry point ccq_fwd_bwd.  Returns 0 for an invalid shape. */
size_t ccq_workspace_size(const ccq_shape* s, ccq_backbone bb, int with_bwd);

/*
 * CCQ-GLA chunkwise forward (Alg. 1 with the GLA chunk form as BackboneUpdate).
 *   q, k     [B,T,H,dk] io_dtype      queries / keys
 *   v        [B,T,H,dv] io_dtype      values
 *   g        [B,T,H,dk] gate_dtype    per-key-channel log forget gate (<= 0)
 *   lam      [B,T,H]    fp32          contraction gate lambda_t (Eq. clean)
 *   S0       [B,H,dv,dk] fp32 or NULL initial backbone state (NULL = 0)
 *   C0       [B,H,dk,dk] fp32 or NULL initial Cbar (NULL = 0), weight t0
 *   mu0      [B,H,dk]    fp32 or NULL initial mu (NULL = 0), weight t0
 *   o        [B,T,H,dv] io_dtype      output (written)
 *   ST, CT, muT  final (S_T, Cbar_T, mu_T), the inference cache of App. C,
 *                same layouts as S0, C0, mu0; each may be NULL (not wanted)
 *   q_clean_dbg [B,T,H,dk] fp32 or NULL: the cleaned queries, for checking
 */
ccq_status ccq_gla_fwd(const ccq_shape* s, const void* q, const void* k, const void* v,
                       const void* g, const float* lam, const float* S0, const float* C0,
                       const float* mu0, void* o, float* ST, float* CT, float* muT,
                       float* q_clean_dbg, void* workspace, size_t ws_bytes, void* stream);

/*
 * CCQ-Gated-DeltaNet chunkwise forward (Alg. 1 with the delta-rule chunk form
 * computed through the WY/UT transform as BackboneUpdate).
 *   logalpha [B,T,H] fp32   log of the per-head scalar decay alpha_t (<= 0)
 *   beta     [B,T,H] fp32   write strength beta_t in [0,1]
 * All other arguments as in ccq_gla_fwd.
 */
ccq_status ccq_gdn_fwd(const ccq_shape* s, const void* q, const void* k, const void* v,
                       const float* logalpha, const float* beta, const float* lam,
                       const float* S0, const float* C0, const float* mu0, void* o, float* ST,
                       float* CT, float* muT, float* q_clean_dbg, void* workspace,
                       size_t ws_bytes, void* stream);

/*
 * Allocation-free form of ccq_gdn_fwd, for callers that cannot allocate device
 * memory or pass a workspace: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Same arguments and results as
 * ccq_gdn_fwd without the workspace: the kernels use a scratch array of
 * CCQ_NOALLOC_SCRATCH_BYTES that the library holds in device memory, one copy
 * per device, from the first call on that device until the process ends.  The
 * call allocates nothing (no hipMalloc, hipFree or allocating library call).
 * Shapes whose ccq_workspace_size(s, CCQ_GDN, 0) exceeds
 * CCQ_NOALLOC_SCRATCH_BYTES return CCQ_ERR_WORKSPACE before anything is
 * launched (at dk = dv = 256 that is about 10,000 token-heads, B*T*H, per call).
 * All calls on one device share its scratch: calls that may overlap on one
 * device (two streams, two host threads) race and must be ordered by the
 * caller; calls ordered on one stream are safe.  The scratch keeps the last
 * call's contents, and no call reads what an earlier call left there.
 */
#define CCQ_NOALLOC_SCRATCH_BYTES ((size_t)64 << 20)
ccq_status ccq_gdn_fwd_noalloc(const ccq_shape* s, const void* q, const void* k, const void* v,
                               const float* logalpha, const float* beta, const float* lam,
                               const float* S0, const float* C0, const float* mu0, void* o,
                               float* ST, float* CT, float* muT, float* q_clean_dbg,
                               void* stream);

/*
 * Training step: forward and the gradients of L = sum_t <dO_t, o_t> with
 * respect to q, k, v, the gates and lambda (fresh sequence: zero initial
 * states, t0 must be 0).
 *   bb = CCQ_GLA: g_or_logalpha is g [B,T,H,dk] gate_dtype; beta and dbeta NULL;
 *                 dg_or_dlogalpha is dg [B,T,H,dk] gate_dtype.
 *   bb = CCQ_GDN: g_or_logalpha is log alpha [B,T,H] fp32 and beta [B,T,H]
 *                 fp32 is required; dg_or_dlogalpha is d(log alpha) [B,T,H]
 *                 fp32 and dbeta [B,T,H] fp32 is required.  The backbone
 *                 gradients follow the reverse of the chunk form through the
 *                 WY/UT transform (Alg. 1's BackboneUpdate for the delta rule).
 *   dO [B,T,H,dv] io_dtype upstream gradient; o, dq, dk, dv io_dtype;
 *   dlam [B,T,H] fp32.
 * Supported: chunk = 64, dv in {64,128,256,512}, and dk in {64,128} for bf16
 * io (also 256 for CCQ_GDN) or dk = 64 for fp32 io; other shapes return
 * CCQ_ERR_UNSUPPORTED.
 */
ccq_status ccq_fwd_bwd(const ccq_shape* s, ccq_backbone bb, const void* q, const void* k,
                       const void* v, const void* g_or_logalpha, const float* beta,
                       const float* lam, const void* dO, void* o, void* dq, void* dk, void* dv,
                       void* dg_or_dlogalpha, float* dbeta, float* dlam, void* workspace,
                       size_t ws_bytes, void* stream);

/*
 * Recurrent inference, one token per sequence (Alg. 2), on the cache triple
 * of App. C, updated in place:
 *   Cbar <- Cbar + (k k^T - Cbar)/t,  mu <- mu + (k - mu)/t,  t = s->t0 + 1;
 *   q_clean = q - lam (Cbar q - mu (mu . q))   (Cbar q alone when centered = 0);
 *   S <- BackboneUpdate(S; k, v, gates);  o = scale S q_clean.
 * s->T must be 1; s->t0 is the number of tokens already absorbed (the cache of
 * a fresh sequence is all zeros with t0 = 0).  q, k [B,H,dk] and v, o [B,H,dv]
 * in io_dtype (one token, T = 1, of the [B,T,H,d] layout); GLA gate g [B,H,dk]
 * gate_dtype; Gated DeltaNet log alpha and beta [B,H] fp32 (beta NULL for GLA);
 * lam [B,H] fp32.  S [B,H,dv,dk], C [B,H,dk,dk] and mu [B,H,dk] are fp32,
 * caller-owned, read and overwritten.  Supported: dk in {64,128,256}, dv in
 * {64,128,256,512}, both backbones and both io dtypes.
 * The workspace holds ccq_decode_workspace_size(s) bytes, B*H*dk*4 rounded
 * up when the step is split into two launches (fewer than 256 heads of large
 * caches), else 0, and workspace may then be NULL.
 */
size_t ccq_decode_workspace_size(const ccq_shape* s);
ccq_status ccq_decode(const ccq_shape* s, ccq_backbone bb, const void* q, const void* k,
                      const void* v, const void* g_or_logalpha, const float* beta,
                      const float* lam, float* S, float* C, float* mu, void* o, void* workspace,
                      size_t ws_bytes, void* stream);

/*
 * Pre-processing of one layer's raw queries and keys (Alg. 1: the per-chunk
 * l2 normalisation of Q and K, and the gate Lambda = sigma(Q W_lambda^T +
 * b_lambda) computed from the query before normalisation; Eq. clean):
 *   q[b,t,h,:] = q_raw[b,t,h,:] / max(|q_raw[b,t,h,:]|, 1e-12), k likewise;
 *   lam[b,t,h] = sigmoid(sum_j w_lam[h][j] q_raw[b,t,j] + b_lam[h]),
 * where j runs over all H*dk features of the token's query before the split
 * into heads (head-major).  q_raw, k_raw, q, k [B,T,H,dk] io_dtype; w_lam
 * [H, H*dk] fp32; b_lam [H] fp32; lam [B,T,H] fp32.  q and k may be q_raw and
 * k_raw (in place).  Uses s->B, T, H, dk and io_dtype.  Supported: dk in
 * {64,128,256}, H <= 16, H*dk <= 2048 and H*H*dk <= 16384 (W_lambda is
 * staged on chip); otherwise CCQ_ERR_UNSUPPORTED.  Allocates nothing.
 */
ccq_status ccq_prep(const ccq_shape* s, const void* q_raw, const void* k_raw, const float* w_lam,
                    const float* b_lam, void* q, void* k, float* lam, void* stream);

/*
 * Forward from the raw queries and keys: Alg. 1's per-chunk l2 normalisation
 * of Q and K and the gate Lambda = sigma(Q W_lambda^T + b_lambda) (Eq. clean)
 * folded into the forward, with the results of ccq_prep followed by
 * ccq_gla_fwd (bb = CCQ_GLA) or ccq_gdn_fwd (bb = CCQ_GDN), but without the
 * normalised q and k ever being written: a first pass reads the raw rows once
 * and writes only the per-row scales 1 / max(|x|, 1e-12) and the gate
 * (3 floats per token and head, in the workspace), and every kernel of the
 * forward scales the raw rows as it stages them.
 *   q_raw, k_raw [B,T,H,dk] io_dtype; w_lam [H, H*dk] fp32; b_lam [H] fp32 (as
 *   ccq_prep); v, the gates, S0, C0, mu0, o, ST, CT, muT as in the forward
 *   entry points (beta required for CCQ_GDN, NULL for CCQ_GLA);
 *   lam_out [B,T,H] fp32 or NULL: the gate, if the caller wants it.
 * The workspace holds ccq_fwd_raw_workspace_size(s, bb) bytes (0 for an
 * unsupported shape).  Shape limits are those of both the forward and
 * ccq_prep (H <= 16, H*dk <= 2048, H*H*dk <= 16384); q_clean export is not
 * offered here.
 */
size_t ccq_fwd_raw_workspace_size(const ccq_shape* s, ccq_backbone bb);
ccq_status ccq_fwd_raw(const ccq_shape* s, ccq_backbone bb, const void* q_raw, const void* k_raw,
                       const float* w_lam, const float* b_lam, const void* v,
                       const void* g_or_logalpha, const float* beta, const float* S0,
                       const float* C0, const float* mu0, void* o, float* ST, float* CT, float* muT,
                       float* lam_out, void* workspace, size_t ws_bytes, void* stream);

/*
 * Packed batches of sequences of different lengths: Alg. 1 (and its
 * training step) applied to every sequence on its own, each an independent
 * recurrence with its own states, exactly as if each were a call of its own.
 * Sequence b occupies rows cu_seqlens[b] .. cu_seqlens[b+1] - 1 of the packed
 * tensors: q, k, dq, dk [rows,H,dk] and v, o, dO, dv [rows,H,dv] in io_dtype,
 * the GLA gate g / dg [rows,H,dk] in gate_dtype, Gated DeltaNet log alpha,
 * beta and their gradients [rows,H] fp32, lam / dlam [rows,H] fp32.
 * cu_seqlens is a DEVICE array of B + 1 int32 (0 = cu[0] <= cu[1] <= ...);
 * s->B is the number of sequences and s->T an upper bound on their lengths
 * (a longer sequence is cut at T; the device offsets are not validated by
 * the host: the packed tensors must hold cu[B] rows).  S0, C0, mu0, ST, CT,
 * muT are per sequence, as in the padded calls; a sequence of length 0 with
 * t0 = 0 returns its initial states (or zeros).  The kernels, of the forward
 * and of the training step, read and write the packed rows directly, through
 * the offsets, and walk only each sequence's own chunks.  q_clean export is
 * not offered here.  The workspace holds ccq_varlen_workspace_size(s, bb,
 * with_bwd) bytes (0: unsupported shape).
 * Errors as for the padded entry points; B > 65535 is CCQ_ERR_UNSUPPORTED.
 */
size_t ccq_varlen_workspace_size(const ccq_shape* s, ccq_backbone bb, int with_bwd);
ccq_status ccq_gla_fwd_varlen(const ccq_shape* s, const int32_t* cu_seqlens, const void* q,
                              const void* k, const void* v, const void* g, const float* lam,
                              const float* S0, const float* C0, const float* mu0, void* o,
                              float* ST, float* CT, float* muT, void* workspace, size_t ws_bytes,
                              void* stream);
ccq_status ccq_gdn_fwd_varlen(const ccq_shape* s, const int32_t* cu_seqlens, const void* q,
                              const void* k, const void* v, const float* logalpha,
                              const float* beta, const float* lam, const float* S0,
                              const float* C0, const float* mu0, void* o, float* ST, float* CT,
                              float* muT, void* workspace, size_t ws_bytes, void* stream);
/* Training step on a packed batch (as ccq_fwd_bwd, t0 = 0; as there, the
 * outputs may not overlap the inputs, which are read after outputs are
 * written). */
ccq_status ccq_fwd_bwd_varlen(const ccq_shape* s, ccq_backbone bb, const int32_t* cu_seqlens,
                              const void* q, const void* k, const void* v,
                              const void* g_or_logalpha, const float* beta, const float* lam,
                              const void* dO, void* o, void* dq, void* dk, void* dv,
                              void* dg_or_dlogalpha, float* dbeta, float* dlam, void* workspace,
                              size_t ws_bytes, void* stream);

/*
 * ---- The gated delta rule without the query contraction ----
 *
 *     S_t = alpha_t S_{t-1} (I - beta_t k_t k_t^T) + beta_t v_t k_t^T,   o_t = scale S_t q_t
 *
 * (ccq_gdn_fwd with lambda = 0, without its key statistics), with query/key heads
 * that several value heads share: value head h reads q and k of head h / (HV / HK).
 *   q, k [B,T,HK,dk], v, o [B,T,HV,dv] io_dtype; logalpha, beta [B,T,HV] fp32;
 *   S0, ST [B,HV,dv,dk] fp32 or NULL (zero; not wanted).
 * ST keeps 17 bits of every operand whatever io_dtype is (with bf16 io, the operands
 * of the state's products are taken as a bf16 head and tail: about 4e-6 from the
 * exact state), so the state may be handed from segment to segment and to
 * ccq_delta_step.  ST may be S0; otherwise outputs may not overlap inputs.  o and the
 * gradients carry bf16 products where io_dtype is bf16 (2.5e-3 to 3.5e-3 of their norm);
 * with T <= 64 and B T HV <= 128 the gradients are formed in fp32, since a norm over so
 * few numbers does not average the products' errors out.  logalpha below -104, -infinity
 * included, is a reset (alpha = 0); the decays between tokens are good to fp32 whatever
 * resets stand ahead of them.
 * Packed batches as for ccq_gdn_fwd_varlen: [rows, heads, d] tensors, device offsets
 * cu_seqlens of B + 1 int32, s->T a bound on the lengths; rows behind cu[B] (and
 * behind a sequence's first T) are not written.  An infinity or NaN among a token's
 * inputs reaches the outputs of its whole chunk of 64 tokens and of those behind it
 * (ccq_delta_step: of the tokens behind it), never another sequence or head.
 * Supported: dv in {64,128,256,512}; dk in {64,128,256} (bf16 io) or {64,128} (fp32
 * io); the training step with fp32 io: dk = 64; ccq_delta_step: dk in {64,128,256},
 * both types.  B > 65535 packed is CCQ_ERR_UNSUPPORTED, and so are sizes that a launch
 * cannot count: HV max(dk, dv) above 2^24; B HV ceil(T / 64) from 2^23 on, and B HV dv
 * from 2^29 (dk = 256: 2^28) on; for ccq_delta_step B HV dv from 2^28 on.
 */
typedef struct {
  int32_t B, T;         /* sequences, tokens (or the bound on them); >= 0 */
  int32_t HK, HV;       /* query/key heads, value heads: HV a multiple of HK */
  int32_t dk, dv;
  ccq_dtype io_dtype;
  float scale;
} ccq_delta_shape;

/* Bytes of workspace of the forward (with_bwd = 0) or the training step; 0: unsupported. */
size_t ccq_delta_workspace_size(const ccq_delta_shape* s, int with_bwd);
ccq_status ccq_delta_fwd(const ccq_delta_shape* s, const void* q, const void* k, const void* v,
                         const float* logalpha, const float* beta, const float* S0, void* o,
                         float* ST, void* workspace, size_t ws_bytes, void* stream);
ccq_status ccq_delta_fwd_varlen(const ccq_delta_shape* s, const int32_t* cu_seqlens, const void* q,
                                const void* k, const void* v, const float* logalpha,
                                const float* beta, const float* S0, void* o, float* ST,
                                void* workspace, size_t ws_bytes, void* stream);
/*
 * Training step: the gradients of L = sum_t <dO_t, o_t>, and o (NULL: not wanted, as
 * where the forward has been run and dO came from what follows it) and ST (NULL: not
 * wanted).  No gradient flows to S0 or from ST.  dq, dk [B,T,HK,dk] (summed over
 * the value heads that share them, in fp32 and in order), dv [B,T,HV,dv],
 * dlogalpha, dbeta [B,T,HV], all io_dtype.  Outputs may not overlap inputs.
 */
ccq_status ccq_delta_fwd_bwd(const ccq_delta_shape* s, const void* q, const void* k, const void* v,
                             const float* logalpha, const float* beta, const float* S0,
                             const void* dO, void* o, float* ST, void* dq, void* dk, void* dv,
                             void* dlogalpha, void* dbeta, void* workspace, size_t ws_bytes,
                             void* stream);
ccq_status ccq_delta_fwd_bwd_varlen(const ccq_delta_shape* s, const int32_t* cu_seqlens,
                                    const void* q, const void* k, const void* v,
                                    const float* logalpha, const float* beta, const float* S0,
                                    const void* dO, void* o, float* ST, void* dq, void* dk,
                                    void* dv, void* dlogalpha, void* dbeta, void* workspace,
                                    size_t ws_bytes, void* stream);
/* The recurrent form for one or a few tokens (s->T of them) per sequence, on the
 * state S [B,HV,dv,dk] fp32, updated in place; fp32 arithmetic; no workspace. */
ccq_status ccq_delta_step(const ccq_delta_shape* s, const void* q, const void* k, const void* v,
                          const float* logalpha, const float* beta, float* S, void* o,
                          void* stream);

/* Activations of the two operators below. */
typedef enum { CCQ_ACT_NONE = 0, CCQ_ACT_SILU = 1, CCQ_ACT_SIGMOID = 2 } ccq_act;

/*
 * ---- Short causal convolution (what q, k and v pass before the recurrence) ----
 *
 *     y_t = act(bias + sum_{j<W} w_j x_{t-W+1+j})       every channel on its own
 *
 *   x [B,T,C] io_dtype, token pitch ldx elements (so a slice of a wider projection
 *   can be read where it lies); w [C,W] fp32; bias [C] fp32 or NULL; y [B,T,C]
 *   io_dtype, dense.  state0 [B,W-1,C] io_dtype: the W - 1 inputs before the first
 *   token, oldest first (NULL: zeros); stateT the same after the last one (NULL: not
 *   wanted).  y and stateT may not overlap x, state0 or each other: a token's inputs are
 *   read by what follows it too (CCQ_ERR_INVALID_ARG; of x and y in a packed batch, whose
 *   rows the host does not know, the caller sees to it).
 * Supported: W in {2,3,4}, C a positive multiple of 8 up to 2^24, ldx >= C with ldx elements a
 * multiple of 16 bytes.  Packed batches: x, y [rows,C], offsets and T as above.
 */
typedef struct {
  int32_t B, T, C, W;
  ccq_dtype io_dtype;
  ccq_act act;
  int64_t ldx;
} ccq_conv_shape;

ccq_status ccq_conv_fwd(const ccq_conv_shape* s, const void* x, const float* w, const float* bias,
                        const void* state0, void* y, void* stateT, void* stream);
ccq_status ccq_conv_fwd_varlen(const ccq_conv_shape* s, const int32_t* cu_seqlens, const void* x,
                               const float* w, const float* bias, const void* state0, void* y,
                               void* stateT, void* stream);
/* Gradients: dy [B,T,C] io_dtype, dense; dstateT [B,W-1,C] io_dtype or NULL (zeros), the
 * gradient of stateT; dx [B,T,C] io_dtype, dense; dw [C,W], dbias [C] fp32 (dbias with
 * bias only, else NULL); dstate0 [B,W-1,C] io_dtype or NULL (not wanted).  Outputs may
 * not overlap inputs.  workspace: ccq_conv_workspace_size(s) bytes (0: unsupported). */
size_t ccq_conv_workspace_size(const ccq_conv_shape* s);
ccq_status ccq_conv_bwd(const ccq_conv_shape* s, const void* x, const float* w, const float* bias,
                        const void* state0, const void* dy, const void* dstateT, void* dx,
                        float* dw, float* dbias, void* dstate0, void* workspace, size_t ws_bytes,
                        void* stream);
ccq_status ccq_conv_bwd_varlen(const ccq_conv_shape* s, const int32_t* cu_seqlens, const void* x,
                               const float* w, const float* bias, const void* state0,
                               const void* dy, const void* dstateT, void* dx, float* dw,
                               float* dbias, void* dstate0, void* workspace, size_t ws_bytes,
                               void* stream);
/* One token per sequence (s->T must be 1): x, y [B,C] (x with pitch ldx); state
 * [B,W-1,C] io_dtype, moved on by the token in place; x, y and state may not overlap. */
ccq_status ccq_conv_step(const ccq_conv_shape* s, const void* x, const float* w, const float* bias,
                         void* state, void* y, void* stream);

/*
 * ---- Group norm of the heads with an activation, channels last ----
 *
 * x is [rows, G, D] (a token's G heads of D channels): every head of every token is
 * normalised on its own,
 *   CCQ_NORM_GROUP  n = (x - mean x) / sqrt(var x + eps)
 *   CCQ_NORM_RMS    n = x / sqrt(mean x^2 + eps)
 *   CCQ_NORM_L2     n = x / sqrt(sum x^2 + eps)
 * then z = n w + bias and y = z act(gate) with a gate, y = act(z) without.
 *   x, gate [rows,G,D] io_dtype with row pitches ldx, ldg elements (a row's G D elements
 *   are dense); w, bias [G,D] fp32, or [D] with shared = 1 (all heads take the same),
 *   or NULL (ones, zeros; bias only with w); gate may be NULL; y [rows,G,D] io_dtype.
 * Supported: D a multiple of 8 up to 8192, G D <= 2^24; ldx, ldg >= G D and a multiple of 16
 * bytes (ldg is read with a gate only); eps >= 0.
 */
typedef enum { CCQ_NORM_GROUP = 0, CCQ_NORM_RMS = 1, CCQ_NORM_L2 = 2 } ccq_norm_kind;
typedef struct {
  int64_t rows;
  int32_t G, D;
  ccq_dtype io_dtype;
  ccq_norm_kind kind;
  ccq_act act;
  int32_t shared;
  float eps;
  int64_t ldx, ldg;
} ccq_norm_shape;

/* y may not overlap x or gate. */
ccq_status ccq_norm_fwd(const ccq_norm_shape* s, const void* x, const float* w, const float* bias,
                        const void* gate, void* y, void* stream);
/* Gradients: dy [rows,G,D] io_dtype, dense; dx, dgate [rows,G,D] io_dtype, dense (dgate with
 * a gate only); dw, dbias fp32, shaped as w and bias (with them only; a shared weight's
 * gradient is summed over the heads).  Outputs may not overlap inputs.  workspace:
 * ccq_norm_workspace_size(s) bytes (0: unsupported), needed with w only. */
size_t ccq_norm_workspace_size(const ccq_norm_shape* s);
ccq_status ccq_norm_bwd(const ccq_norm_shape* s, const void* x, const float* w, const float* bias,
                        const void* gate, const void* dy, void* dx, float* dw, float* dbias,
                        void* dgate, void* workspace, size_t ws_bytes, void* stream);

/*
 * Per-kernel timing hook (instrumentation for benchmarks and profilers, not
 * part of the method).  `events` points at n_events hipEvent_t handles created
 * by the caller (hipEventCreate).  Until the next ccq_trace_events call from
 * the same host thread, every entry point called from that thread records
 * events[2i] on its stream just before its i-th kernel launch and
 * events[2i+1] just after it, for i < n_events/2; the count restarts at each
 * entry-point call.  events = NULL (or n_events = 0) switches tracing off.
 * The setting is per host thread; nothing else is kept between calls.
 */
ccq_status ccq_trace_events(void* const* events, int n_events);

/* Human-readable text of a status code (static storage). */
const char* ccq_status_string(ccq_status st);

/* Library version string, e.g. "ccq-mi355x 0.1.0 gfx950". */
const char* ccq_version(void);

#ifdef __cplusplus
}
#endif

#endif /* CCQ_H_ */
