/*
 * tsfm.h -- C ABI of the B200 (sm_100a) speculative decoder for continuous patch
 * autoregression.
 *
 * The library decodes a batch of univariate series patch by patch with a decoder-only
 * patch transformer ("target"), optionally accelerated by a cheap draft model under the
 * Gaussian speculative-decoding rule:
 *
 *   - patch-autoregressive decoding, T = ceil(H / P) patches per series   (paper Eq. 1)
 *   - Gaussian surrogate heads N(mu, sigma^2 I) with a supplied shared
 *     scale sigma, here called `tau`                                      (Sec. 3.1, Eq. 4)
 *   - acceptance statistic l_i = (1/d) log p(x_i)/q(x_i), accept with
 *     probability min{1, exp(l_i)}, evaluated in the log domain           (Sec. 3.2, Eq. 5)
 *   - mean proposals x_i = mu_q^(i), target-mean fallback, bonus patch    (Sec. 3.3, Eq. 6)
 *   - single causal verification pass over [h, x_1..x_K], read at the
 *     K+1 prefix boundaries; instance statistics frozen on the context    (Sec. 3.4)
 *   - one round = Algorithm 1 (appendix B), looped until T patches are committed.
 *
 * Conventions
 *   - "dev" pointers are CUDA device pointers on the current device; "host" pointers are
 *     ordinary host memory.  Nothing in this ABI is a torch type.
 *   - All work is enqueued on the stream given at creation (a cudaStream_t passed as void*,
 *     NULL = the legacy default stream).  Calls that return data to host memory (stats,
 *     traces) synchronise that stream before returning; the others are asynchronous.
 *   - Every function returns 0 on success or a negative TSFM_ERR_* code.  Nothing aborts,
 *     traps, or throws across this boundary.  Device-side waits are bounded; if one expires
 *     the call returns TSFM_ERR_TIMEOUT and the CUDA context stays usable.
 *   - There is no CPU fallback: on a machine without an sm_100 device every compute entry
 *     point returns TSFM_ERR_ARCH / TSFM_ERR_CUDA.
 */
#ifndef TSFM_H_
#define TSFM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define TSFM_OK            0
#define TSFM_ERR_ARG      (-1)  /* null pointer, B < 1, K < 1, tau not finite or <= 0, H < 1           */
#define TSFM_ERR_SHAPE    (-2)  /* ctx_len % P != 0, fewer than 2 context patches, capacity exceeded
                                   (B, N, T or K beyond the handle's max_*), d_model % n_heads != 0,
                                   unsupported head size, bad weight blob                           */
#define TSFM_ERR_ARCH     (-3)  /* current device is not compute capability 10.x                   */
#define TSFM_ERR_CUDA     (-4)  /* a CUDA runtime/driver call failed (see tsfm_last_cuda_error)     */
#define TSFM_ERR_TIMEOUT  (-5)  /* a bounded device-side wait expired                               */
#define TSFM_ERR_INTERNAL (-6)

#define TSFM_F32   0            /* weights, activations and KV cache in fp32 (SIMT FMA path)        */
#define TSFM_BF16  1            /* bf16 weights / MMA operands / KV cache, fp32 accumulate+residual */

#define TSFM_DRAFT_SEPARATE   0 /* draft has its own weight blob                                    */
#define TSFM_DRAFT_LAYER_SKIP 1 /* draft = first draft.n_layers layers of the target + its final
                                   norm and head; draft_w must be NULL                              */

#define TSFM_GEMM_AUTO  0       /* bf16 contractions on tcgen05 tensor cores where shapes allow     */
#define TSFM_GEMM_SIMT  1       /* force the plain FMA kernels everywhere (differential reference)  */
#define TSFM_GEMM_WS    2       /* tsfm_gemm_bf16 only: the small-batch kernel that keeps its weight
                                   tile in registers (TSFM_ERR_SHAPE outside its domain: at most
                                   512 tokens, K a multiple of 64 up to 2048, N even, a grid of
                                   16 x 32 tiles that is resident at once,
                                   C 8-byte aligned);
                                   a decoder picks it by itself where it applies                   */

#define TSFM_EXEC_GRAPH   0       /* a forecast is one CUDA-graph launch: prologue, a device-side WHILE
                                   over the rounds, de-normalisation; no host round trip             */
#define TSFM_EXEC_STREAM  1       /* kernels are launched one by one and the host checks for completion
                                   after every round (reference behaviour; also used while profiling) */

#define TSFM_EXEC_NO_PDL  2       /* flag, may be OR-ed in: launch without programmatic dependent launch,
                                   i.e. every kernel starts only after its predecessor has finished   */

#define TSFM_EXEC_NO_COMPACT 4     /* flag, may be OR-ed in: every round runs its passes over all B series, finished
                                   or not (by default only the series that still have patches to commit take
                                   part: the batch desynchronises as per-series first rejections differ, the
                                   paper's "Batch Size" sensitivity paragraph); same results either way  */

#define TSFM_EXEC_CHECK_BOUNDS 8   /* flag, may be OR-ed in: bounds-checking mode.  Every device buffer of the handle
                                   gets guard bytes behind it, every (layer, series, head) block of the KV
                                   caches and every series' history one spare token that nothing may write;
                                   after each call a kernel inspects them all, and a damaged guard makes a
                                   call that reads its status (stats != NULL) return TSFM_ERR_INTERNAL with
                                   the buffer's name in tsfm_last_cuda_error().  Costs memory and a launch
                                   per call; for test runs                                               */

#define TSFM_MAX_K 32           /* hard upper bound on the block size K                             */

typedef struct tsfm_spec tsfm_spec;   /* opaque decoder handle */

/* Decoder-only pre-norm patch transformer: n_layers x {RMSNorm, RoPE causal attention with
 * n_heads heads, RMSNorm, GELU MLP d_model -> d_ff -> d_model}, linear patch embedding and
 * linear mean head.  d_model % n_heads == 0; head size d_model / n_heads in {32, 64, 128};
 * d_model and d_ff multiples of 64; patch_len a multiple of 16, at most 256. */
typedef struct {
  int32_t n_layers, d_model, n_heads, d_ff;
} tsfm_arch;

typedef struct {
  tsfm_arch target, draft;
  int32_t patch_len;            /* P: input and output patch length (one channel)               */
  int32_t dtype;                /* TSFM_F32 | TSFM_BF16                                          */
  int32_t draft_mode;           /* TSFM_DRAFT_*                                                  */
  int32_t max_batch;            /* capacity: series per call                                     */
  int32_t max_ctx_tokens;       /* capacity: context tokens N = ctx_len / P_in (>= 2 patches' worth) */
  int32_t max_horizon_patches;  /* capacity: T = ceil(H / P)                                     */
  int32_t max_K;                /* capacity: block size, <= TSFM_MAX_K                           */
  int32_t gemm_backend;         /* TSFM_GEMM_*                                                   */
  float   rms_eps;              /* RMSNorm epsilon (1e-6)                                        */
  float   norm_eps;             /* instance-norm variance epsilon (1e-5)                         */
  float   rope_base;            /* RoPE base (1e4)                                               */
  int32_t exec_mode;            /* TSFM_EXEC_GRAPH or TSFM_EXEC_STREAM, optionally | TSFM_EXEC_NO_PDL | TSFM_EXEC_NO_COMPACT */
  int32_t patch_in;             /* P_in: steps per INPUT token; 0 = patch_len (a token is a whole patch).
                                   Must divide patch_len.  With P_in < P (the point-token family of the
                                   paper's appendix B: P_in = 1, a horizon head of P steps) a committed
                                   patch is P / P_in tokens, the embedding is [d, P_in], and the target's
                                   prediction after prefix i is read at token N - 1 + i (P / P_in) of the
                                   verification pass (appendix B, "Per-Family Boundary Indexing")        */
  void   *stream;               /* cudaStream_t, borrowed for the handle's lifetime              */
} tsfm_cfg;

/* A weight blob in DEVICE memory, borrowed for the handle's lifetime (never copied, never
 * written).  Layout: a 256-byte header of int32 words
 *     [0] magic 0x4D465354 ("TSFM")  [1] version 1  [2] dtype  [3] n_layers  [4] d_model
 *     [5] n_heads  [6] d_ff  [7] patch_len  [8] patch_in (0 = patch_len)   (remaining words zero)
 * followed by the tensors, each starting on a 256-byte boundary, every linear stored
 * [out_features, in_features] row-major in `dtype`, gains in fp32, in this order:
 *     W_emb[d,P_in];  per layer: g1[d], Wq[d,d], Wk[d,d], Wv[d,d], Wo[d,d], g2[d],
 *     W1[d_ff,d], W2[d,d_ff];  g_f[d];  W_head[P,d].
 * tsfm_weights_bytes() gives the total size. */
typedef struct {
  const void *blob;             /* dev */
  size_t      bytes;
} tsfm_weights;

/* Counters of one forecast call (host memory).  "tested" counts proposals whose accept/reject
 * decision was taken (accepted ones plus the first rejected one of each round): accepted/tested
 * estimates the conditional acceptance rate of the capped-geometric law (Eq. 7). */
typedef struct {
  int64_t rounds;                       /* speculative rounds executed (max over series)        */
  int64_t proposals_drafted;            /* K per active series per round                        */
  int64_t proposals_tested;
  int64_t proposals_accepted;
  int64_t patches_committed;            /* after truncation to T; equals B * T on success       */
  int64_t near_margin_decisions;        /* tested decisions with |l_i - log u_i| < margin       */
  int64_t tested_by_pos[TSFM_MAX_K];
  int64_t accepted_by_pos[TSFM_MAX_K];
  int64_t L_hist[TSFM_MAX_K + 2];       /* untruncated round yield L = n_accept + 1, index L    */
  float   ms_total, ms_prefill, ms_draft, ms_verify, ms_accept;   /* CUDA-event times           */
  int32_t device_status;                /* 0, or the code a kernel's bounded wait reported      */
  int32_t reserved0;
} tsfm_stats;

/* Size in bytes of the weight blob of a model of this shape. Returns 0 on invalid arguments. */
size_t tsfm_weights_bytes(const tsfm_arch *arch, int32_t patch_len, int32_t dtype);

/* Byte offset of a tensor inside the blob; `layer` is ignored for W_emb (-1), g_f, W_head.
 * `name` is one of "W_emb","g1","Wq","Wk","Wv","Wo","g2","W1","W2","g_f","W_head".
 * Returns 0 on invalid arguments (no tensor lives at offset 0: the header does). */
size_t tsfm_weights_offset(const tsfm_arch *arch, int32_t patch_len, int32_t dtype,
                           int32_t layer, const char *name);

/* The same two queries for a model whose input tokens are patch_in steps long (0 = patch_len):
 * only W_emb [d, patch_in] differs.  Return 0 if patch_in does not divide patch_len. */
size_t tsfm_weights_bytes_io(const tsfm_arch *arch, int32_t patch_in, int32_t patch_len, int32_t dtype);
size_t tsfm_weights_offset_io(const tsfm_arch *arch, int32_t patch_in, int32_t patch_len, int32_t dtype,
                              int32_t layer, const char *name);

/* Create a decoder (Algorithm 1's inputs "target p, draft q").  Validates shapes and blob
 * headers, allocates both KV caches ([layer][series][head][token][d_head], capacity
 * max_ctx_tokens + (max_horizon_patches + max_K + 1) * (P / P_in) tokens per series), activation workspaces
 * and TMA descriptors.  target_w, cfg, out_h: host pointers to structs; blobs: dev.
 * draft_w may be NULL only with TSFM_DRAFT_LAYER_SKIP.  *out_h is owned by the caller and
 * released with tsfm_spec_destroy. */
int tsfm_spec_create(const tsfm_weights *target_w, const tsfm_weights *draft_w,
                     const tsfm_cfg *cfg, tsfm_spec **out_h);

/* Speculative forecast (Algorithm 1 looped; Sec. 3.1-3.4).
 *   series  dev  [B, ctx_len] fp32 row-major, raw (un-normalised) context values
 *   out     dev  [B, H] fp32 row-major, forecast in the series' own scale
 *   stats   host, nullable; when non-NULL the call synchronises the stream and fills it
 * ctx_len must be a multiple of P (hence of P_in) with at least 2 patches; T = ceil(H / P) patches are
 * committed per series, the last one truncated to H on output.  Each round drafts K patches
 * with the draft model, verifies them in one causal target pass, accepts left to right with
 * uniforms Philox4x32-10(key = seed, counter = (series, round, position, 0)), commits the
 * accepted proposals plus the target's correction or bonus patch, and rolls both KV caches
 * back to the committed length.  tau is the acceptance temperature (the paper's sigma). */
int tsfm_spec_forecast(tsfm_spec *h, const float *series, int32_t B, int32_t ctx_len,
                       int32_t H, int32_t K, float tau, uint64_t seed,
                       float *out, tsfm_stats *stats);

/* The general form of the rule (Sec. 3.3 "Fallback Correction and Sampled Variants", Algorithm 1
 * with r > 0; component ablation of Table 2).  The deployed scheme is tsfm_spec_forecast: mean
 * proposals, r = 0, sigma_q = sigma_p = tau, 1/d tempering.
 *   sigma_q           draft surrogate scale of Eq. 5; 0 = same as tau (determinant term vanishes)
 *   fallback_noise    r >= 0: correction and bonus patches are mu_p + r eps
 *   sample_proposals  nonzero: x_i = mu_q^(i) + sigma_q eps, the draft continues from the sampled x_i
 *   no_tempering      nonzero: drop the 1/d factor of the statistic
 * eps are standard normals from the same Philox key: Box-Muller on the words of counter
 * (series, round, position, stream | element / 2), stream 0x10000000 for proposals and 0x20000000
 * for the fallback, cosine branch for even elements, sine for odd.  variant == NULL is the deployed
 * scheme. */
typedef struct {
  float   sigma_q;
  float   fallback_noise;
  int32_t sample_proposals;
  int32_t no_tempering;
} tsfm_variant;
int tsfm_spec_forecast_variant(tsfm_spec *h, const float *series, int32_t B, int32_t ctx_len,
                               int32_t H, int32_t K, float tau, uint64_t seed,
                               const tsfm_variant *variant, float *out, tsfm_stats *stats);

/* Target-only decoding (Eq. 1): T sequential one-token target passes.  Same argument
 * meaning as above; only the timing fields, rounds (= T) and patches_committed of `stats`
 * are filled. */
int tsfm_target_only_forecast(tsfm_spec *h, const float *series, int32_t B, int32_t ctx_len,
                              int32_t H, float *out, tsfm_stats *stats);

/* Draft-only decoding: the same loop as tsfm_target_only_forecast run with the draft model alone
 * (the third arm of the paper's matched three-way protocol, Sec. 4.1 "Evaluation Protocol").
 * Timing goes to ms_prefill / ms_draft. */
int tsfm_draft_only_forecast(tsfm_spec *h, const float *series, int32_t B, int32_t ctx_len,
                             int32_t H, float *out, tsfm_stats *stats);

/* The two forecasts with HOST buffers: series host [B, ctx_len], out host [B, H] (pinned
 * memory makes the copies asynchronous; pageable memory works too).  The input is copied to
 * a device staging buffer owned by the handle, the forecast runs as above, the result is
 * copied back, and the stream is synchronised before returning. */
int tsfm_spec_forecast_host(tsfm_spec *h, const float *series, int32_t B, int32_t ctx_len,
                            int32_t H, int32_t K, float tau, uint64_t seed,
                            float *out, tsfm_stats *stats);
int tsfm_target_only_forecast_host(tsfm_spec *h, const float *series, int32_t B, int32_t ctx_len,
                                   int32_t H, float *out, tsfm_stats *stats);

/* Per-round decisions of the last tsfm_spec_forecast on this handle, copied to HOST arrays
 * (any may be NULL).  R = rounds of that call, B and K as in that call.
 *   n_accept [R, B] int32: leading accepted proposals, or -1 if the series had finished
 *   ell      [R, B, K] fp32: l_i of Eq. 5 for every position (tested or not)
 *   log_u    [R, B, K] fp32: log of the uniform drawn for that position
 * *rounds receives R.  cap_rounds is the first dimension of the arrays the caller provided;
 * returns TSFM_ERR_ARG if it is smaller than R.  Synchronises the stream. */
int tsfm_spec_last_trace(tsfm_spec *h, int32_t cap_rounds, int32_t *rounds,
                         int32_t *n_accept, float *ell, float *log_u);

/* One fused accept step (Eq. 5 + first rejection + correction/bonus) on caller buffers, the
 * same kernel the round uses.  All pointers dev.
 *   x     [B, K, P]   proposals x_i            mu_q [B, K, P] draft means (may alias x)
 *   mu_p  [B, K+1, P] boundary predictions
 *   done  [B] int32   in/out: patches committed so far; series with done >= T are skipped
 *   commit[B, K+1, P] out: x_1..x_n then mu_p^(n+1)          n_accept [B] int32 out
 *   ell, log_u [B, K] out (nullable)
 * sigma_p, sigma_q: the two surrogate scales (equal in the deployed scheme); round_idx and
 * series0 enter the Philox counter; forced_u (dev [B, K], nullable) replaces the drawn
 * uniforms, for scripted tests. */
int tsfm_accept_round(void *stream, const float *x, const float *mu_q, const float *mu_p,
                      int32_t B, int32_t K, int32_t P, int32_t T, float sigma_p, float sigma_q,
                      uint64_t seed, int32_t round_idx, int32_t series0, const float *forced_u,
                      int32_t *done, float *commit, int32_t *n_accept, float *ell, float *log_u);

/* Full causal forward of one of the handle's models over fresh sequences (positions
 * 0..n-1), for numerics checks: tokens dev [B, n, P_in] fp32 (already normalised), out dev
 * [B, n, P] fp32 = next-patch mean at every position.  which: 0 target, 1 draft.
 * n <= max_ctx_tokens (TSFM_ERR_SHAPE beyond it).  Overwrites the KV cache; synchronises the stream. */
int tsfm_model_forward(tsfm_spec *h, int32_t which, const float *tokens, int32_t B, int32_t n,
                       float *out);

/* C[M, N] = A[M, Kd] * W[N, Kd]^T with bf16 operands and fp32 accumulation, through the
 * tensor-memory kernel (backend TSFM_GEMM_AUTO), the FMA kernel (TSFM_GEMM_SIMT) or the small-batch
 * kernel (TSFM_GEMM_WS); for differential tests of the contraction.  A, W dev bf16 row-major; C dev fp32 row-major. */
int tsfm_gemm_bf16(void *stream, const void *A, const void *W, float *C,
                   int32_t M, int32_t N, int32_t Kd, int32_t backend);

/* The same contraction as tsfm_gemm_bf16 (tensor-core kernel, K split across CTAs with fp32
 * atomic accumulation) for callers that must not allocate device memory.  The paper has no
 * counterpart to this entry point; it exists for the library's users.  Who they are: a
 * serving loop that checks the contraction while forecasts are in flight on other streams
 * (cudaMalloc and cudaFree synchronise the whole device and would stall those forecasts), and
 * a process that has handed all device memory to a pooling allocator, where a raw cudaMalloc
 * can simply fail.  This call makes no cudaMalloc, cudaFree or other allocating call.
 *   - Scratch (the split-K accumulator and a status word) is a fixed array of
 *     256 + 4 * TSFM_STATIC_GEMM_MAX_ELEMS bytes (4 MiB + 256 B) inside the library image; every
 *     GPU that loads the library holds it until the process exits.
 *   - M * N must not exceed TSFM_STATIC_GEMM_MAX_ELEMS: larger outputs are rejected with
 *     TSFM_ERR_SHAPE and a message available from tsfm_last_cuda_error().
 *   - The first call on each device looks up the array's device address; make that first call
 *     outside of any stream capture.
 *   - Every call on a device shares the one array, which still holds the previous call's
 *     contents: the call clears the part it uses before accumulating.  Two calls that overlap
 *     on the GPU (different streams, or threads) race on it; serialise them.
 * A, W dev bf16 row-major, C dev fp32 [M, N] row-major (written last, by a device-to-device
 * copy); synchronises `stream` before returning. */
#define TSFM_STATIC_GEMM_MAX_ELEMS (1 << 20)
int tsfm_gemm_bf16_static(void *stream, const void *A, const void *W, float *C,
                          int32_t M, int32_t N, int32_t Kd);

/* ---------------------------------------------------------------------------------------------
 * Serving over a cache of pages.
 *
 * A decoder handle keeps one contiguous cache block of full capacity per series.  The calls below
 * are the steps of a round for callers that manage the cache themselves, as a server of many
 * series or of a model over quantised values (tokens) does: append the new tokens' keys and values
 * with their rotary positions, attend the new tokens to the cache, verify drafted tokens, and, for
 * streams that never end, evict what got little attention.  As in a decoder every cache position
 * derives from the committed length len[b], which only tsfm_verify_tokens (and tsfm_cache_evict)
 * moves: the round's tokens lie in slots len[b] .. len[b] + n_new[b] - 1, and what a verification
 * rejects is garbage behind the new length.
 *
 * A decoder handle does not use these calls, and its norms, MLPs, embeddings and heads are not exported as steps
 * of their own: what lies between an append and a verification is the caller's (tsfm_gemm_bf16 is there for products).
 *
 * All four enqueue kernels on `stream` and return; they allocate nothing, keep nothing between
 * calls, and can be captured into a CUDA graph.  Pointers are dev on the current device unless
 * said otherwise; `stream` belongs to the current device.  Two calls that overlap on the GPU must
 * not share a workspace, nor pages, lengths or counts of tokens that one of them writes.
 *
 * A pool holds pages of page_size slots for all series.  Slot s of series b lies in page
 * table[b * table_stride + s / page_size]; element i of its key for head h is
 *     k[page * page_stride + h * head_stride + (s % page_size) * slot_stride + i]
 * (strides in elements), its value likewise in v.  Page ids are read up to the series' length
 * only.  Device data that is wrong does not fault: an id outside [0, n_pages) is never
 * followed (its slots are hidden from attention, appends to it are dropped, an eviction copies
 * nothing from or to it) and sets TSFM_PAGES_BAD_ID in *status; a length below 0 or beyond the
 * capacity is cut to it (an append drops the tokens that lie outside) and sets TSFM_PAGES_BAD_LEN.
 * *status is only ever OR-ed into.
 *
 * Restrictions (TSFM_ERR_SHAPE): d_head 32, 64 or 128; page_size a power of two up to 65536;
 * pointers to keys, values, queries and outputs and their strides multiples of 16 bytes. */
#define TSFM_PAGES_BAD_ID  1
#define TSFM_PAGES_BAD_LEN 2
#define TSFM_PAGES_TIMEOUT 4    /* a bounded device-side wait expired: outputs that depend on it are NaN */

typedef struct {
  void          *k, *v;         /* dev pools of `dtype`                                         */
  int64_t        page_stride, head_stride, slot_stride;
  const int32_t *table;         /* dev [B, table_stride]; pages of a series in slot order       */
  int32_t        table_stride;
  int32_t        max_pages;     /* entries of a row that may be used: capacity max_pages * page_size */
  int32_t        n_pages;       /* pages in the pool                                            */
  int32_t        page_size;
  int32_t        n_kv_heads, d_head;
  int32_t        dtype;         /* TSFM_F32 | TSFM_BF16, of the cache, the queries and the outputs */
  int32_t       *status;        /* dev, nullable                                                */
} tsfm_kv_pages;

/* Rotary positions.  The leading rot_dim elements of a head turn in pairs: pair i < rot_dim / 2 at
 * position t goes (x, y) -> mscale (x cos a - y sin a, x sin a + y cos a), a = t f_i; the other
 * elements stay.  HALF pairs elements i and i + rot_dim / 2 (the decoder's own layout), INTERLEAVED
 * elements 2 i and 2 i + 1.  Frequencies, for base b and factor F:
 *     PLAIN   f_i = b^(-2 i / rot_dim)
 *     LINEAR  f_i / F                                  (positions divided by F)
 *     BASE    PLAIN with b F^(rot_dim / (rot_dim - 2)) for b
 *     PARTS   f_i (g_i + (1 - g_i) / F), g_i = clamp((n_i - turns_lo) / (turns_hi - turns_lo), 0, 1),
 *             n_i = original_len f_i / (2 pi): frequencies that turn often within the original
 *             context stay, those that turn seldom are divided by F.
 * mscale multiplies the turned elements (1 for none). */
#define TSFM_ROPE_HALF        0
#define TSFM_ROPE_INTERLEAVED 1
#define TSFM_ROPE_PLAIN  0
#define TSFM_ROPE_LINEAR 1
#define TSFM_ROPE_BASE   2
#define TSFM_ROPE_PARTS  3
typedef struct {
  int32_t  layout, rot_dim;
  float    mscale;
  int32_t  reserved0;
  uint64_t turn[64];            /* 2^64 x turns of pair i per position, modulo 2^64               */
} tsfm_rope;

/* Fill *rope (host; host arithmetic only).  TSFM_ERR_ARG: rope NULL, unknown layout or scaling,
 * rot_dim odd, negative or above 128, base or factor not finite or < 1 (base > 1), mscale not finite,
 * BASE with rot_dim 2, PARTS without original_len > 0 and 0 <= turns_lo < turns_hi.  The last
 * three numbers count for PARTS only. */
int tsfm_rope_init(tsfm_rope *rope, int32_t layout, int32_t rot_dim, int32_t scaling, double base, double factor,
                   double original_len, double turns_lo, double turns_hi, float mscale);

/* Turn the queries and keys of up to M new tokens per series and append keys and values to the
 * cache.  Token m < n_new[b] of series b has position pos[b] + m and slot len[b] + m.
 *   qkv     [B, M] rows of (n_heads + 2 n_kv_heads) * d_head elements, qkv_stride elements apart: the
 *           query heads, the key heads, the value heads (one product with stacked weights)
 *   q_out   [B, M] rows of n_heads * d_head, q_out_stride apart: turned queries.  May be qkv itself
 *           (same stride: in place), otherwise disjoint from it; NULL: queries are not touched
 *   pos     [B] position of the first new token; NULL: len (they part once slots are evicted)
 *   len     [B] slots already in the cache; not cut here: a token whose slot is below 0 or beyond the capacity is not
 *           appended (its queries are turned all the same) and sets TSFM_PAGES_BAD_LEN
 *   n_new   [B] new tokens, cut to 0 .. M; NULL: M each.  Rows behind them are not touched
 * rope->rot_dim <= d_head; n_heads >= 0; a row of at most 2^30 elements.  Pages that are written belong to one series only. */
int tsfm_rope_append(void *stream, const tsfm_rope *rope, const tsfm_kv_pages *pages, const void *qkv, int64_t qkv_stride,
                     void *q_out, int64_t q_out_stride, const int32_t *pos, const int32_t *len, const int32_t *n_new,
                     int32_t B, int32_t M, int32_t n_heads);

/* Attention of up to M new tokens per series over the cache.  Token m < n_new[b], head h, reads key
 * head h / (n_heads / n_kv_heads); it sees slots max(0, end - window) <= s < end, where end is
 * len[b] + m + 1 with `causal` (the new tokens are in the cache, each sees those before it and
 * itself) and len[b] without (they are not; encoder caches).  window 0: no lower bound.  |scale| < 2.3e38.
 *   out  softmax(scale q.k) v;  lse  log of the sum of exp(scale q.k).
 * Scores, maxima and sums are fp32 and out is rounded once.  With bf16 the probabilities enter the product with the
 * values as two bf16 parts: 2^-16 of each probability is lost, not 2^-8.  lse and w_out are fp32 throughout.
 * A token that sees nothing (or only scores of -inf) gets out 0, lse -inf.  What lies in slots that a
 * token does not see has no influence, NaN included.  An infinite value in a slot that it sees may come out as NaN.
 *   q, out  [B, M] rows of n_heads * d_head, q_stride / out_stride elements apart
 *   lse     [B, M, n_heads] fp32, nullable
 *   w_out   nullable, [B, n_kv_heads] rows of w_stride fp32: w_out = w_in + the probabilities that a
 *           slot got, summed over the series' new tokens and the heads of the group, for every slot
 *           below len[b] + n_new[b] (len[b] without causal); behind them nothing is written.  w_in NULL
 *           counts as 0 and may be w_out.  A series with n_new[b] <= 0 copies w_in.
 *   max_len the longest series of the call in slots, new tokens included: lengths are cut to it.
 *           It sizes the grid and the workspace, not the work.  w_stride >= max_len
 *   workspace  256-byte aligned, tsfm_paged_attention_workspace() bytes; contents do not matter
 * n_heads is a multiple of n_kv_heads, M n_heads / n_kv_heads at most 65535.  Rows of tokens m >= n_new[b] are not
 * touched.  Results do not depend on the other series' lengths
 * beyond rounding, and are the same each time for the same call.
 * Made for few new tokens: every 8 to 32 (fp32: 1 to 16) of a key head's M n_heads / n_kv_heads rows read all slots that any
 * token of the series sees, also where they belong to tokens m >= n_new[b].  A prompt of thousands of tokens is right but slow
 * (2048 tokens, 32 heads of 128 over 8 key heads: 0.8 ms): tsfm_window_attention, with window 0 if there is none, is made for those (0.1 ms). */
int tsfm_paged_attention(void *stream, const tsfm_kv_pages *pages, const void *q, int64_t q_stride, void *out, int64_t out_stride,
                         const int32_t *len, const int32_t *n_new, int32_t B, int32_t M, int32_t n_heads, float scale,
                         int32_t causal, int32_t window, int32_t max_len, float *lse, const float *w_in, float *w_out,
                         int64_t w_stride, void *workspace, size_t workspace_bytes);

/* Bytes of workspace for a call of this shape (host arithmetic only; of `pages` the shapes and the dtype
 * count).  0 on invalid arguments. */
size_t tsfm_paged_attention_workspace(const tsfm_kv_pages *pages, int32_t B, int32_t M, int32_t n_heads, int32_t max_len,
                                      int32_t with_weights);

/* Tests only, process-wide, not to be called while another thread attends: later calls of tsfm_paged_attention, tsfm_tree_attention
 * and tsfm_window_attention wait at most wait_us (0, or more than the default of 100 ms: the default) for a tile of slots, and with miss_from >= 0 every CTA waits, from that
 * tile of its own on, for more bytes than it copies: the wait runs out, TSFM_PAGES_TIMEOUT is set, what depends on those tiles
 * is NaN, and the call ends.  Pages of less than eight slots are copied by other means and do not wait.  (0, -1) restores. */
void tsfm_debug_tile_wait(int64_t wait_us, int32_t miss_from);

/* Eviction by accumulated weight: per series and key head, the slots to keep become slots 0, 1, .. (in
 * their old order) of the pages that dst_table names, in the same pool.  A series of L = len[b] <=
 * budget slots keeps them all; otherwise the first `sinks`, the last `recent`, and of the slots between
 * them the budget - sinks - recent with the largest w (equal ones: the lower slot; NaN counts as
 * lowest).  Heads keep different slots; keys are stored turned, so attention does not ask where they
 * were.  The old pages are not written: they may be shared, and are the caller's to release.
 *   dst_table [B] rows of dst_stride page ids, at least ceil(budget / page_size) of them readable (up to
 *             the kept slots' last); its pages belong to one series and to no row of pages->table
 *   w         [B, n_kv_heads] rows of w_stride fp32 (as tsfm_paged_attention accumulates them)
 *   max_len   the longest series in slots: lengths are cut to it.  w_stride >= max_len
 *   kept      [B, n_kv_heads, budget] int32 out: old slot of each new one, ascending, -1 behind them
 *   w_out     [B, n_kv_heads] rows of w_out_stride >= budget fp32, nullable: w of the kept slots; not
 *             written behind them.  Must not overlap w
 *   len_out   [B] out: min(L, budget); must not be len
 * budget >= 1, sinks and recent >= 0, sinks + recent <= budget. */
int tsfm_cache_evict(void *stream, const tsfm_kv_pages *pages, const int32_t *dst_table, int32_t dst_stride, const int32_t *len,
                     const float *w, int64_t w_stride, int32_t B, int32_t budget, int32_t sinks, int32_t recent, int32_t max_len,
                     int32_t *kept, float *w_out, int64_t w_out_stride, int32_t *len_out);

/* Verification of drafted tokens: tsfm_accept_round's counterpart for heads that give a distribution
 * over V tokens.  Proposals x_1..x_nd of series b (nd = n_draft[b], or K) are accepted from the left
 * while u_i q_i(x_i) < p_i(x_i), compared exactly; after n acceptances the committed tokens are
 * x_1..x_n and one drawn from r = max(p_{n+1} - q_{n+1}, 0) (n < nd: the first rejection) or r = p_{n+1}
 * (n = nd: the bonus): the smallest t with r_0 + .. + r_t > u_{K+1} (r_0 + .. + r_{V-1}), in fp64.  Where r is 0
 * everywhere r = p_{n+1}.  Entries of p and q that are negative or not finite count as 0, uniforms are
 * cut to [0, 1 - 2^-24], a proposal outside [0, V) is rejected.
 *   tokens  [B, K] int32 proposals
 *   p       [B, K+1] rows of V fp32, p_stride elements apart: the target's probabilities at the boundaries
 *   q       [B, K] rows of V fp32, q_stride apart: the draft's; NULL: proposals without a distribution
 *           (the draft's best token), q_i is 1 at x_i and 0 elsewhere
 *   u       [B, K+1] fp32 uniforms, the last one for the draw; NULL: the Philox uniforms of
 *           tsfm_accept_round, counter (series0 + b, round_idx, position, 0), key = seed
 *   n_draft [B], nullable, cut to 0 .. K; the draw of a series with fewer uses u_{K+1} all the same
 *   out     [B, K+1] int32: the n + 1 committed tokens, -1 behind them (the drawn one is -1 too where p
 *           has no positive entry)
 *   n_accept [B] int32 out
 *   len, len_out  [B] int32, both or neither: len_out = len + n + 1, the committed length; may be the same
 * K <= TSFM_MAX_K, V <= 2^30; K = 0 draws one token.  out overlaps no input. */
int tsfm_verify_tokens(void *stream, const int32_t *tokens, const float *p, int64_t p_stride, const float *q, int64_t q_stride,
                       int32_t B, int32_t K, int32_t V, const float *u, uint64_t seed, int32_t round_idx, int32_t series0,
                       const int32_t *n_draft, const int32_t *len, int32_t *out, int32_t *n_accept, int32_t *len_out);

/* ---------------------------------------------------------------- trees of drafted tokens, windows with sinks, log probabilities
 * A draft may offer several candidates for a place: M nodes of a tree in place of K proposals in a row.  Node 0 is the last
 * committed token, which the target has not seen yet; parent[m] < m is the node that m hangs on (-1: none).  A round: tsfm_tree_init (once
 * for a tree, whatever the number of layers; a tree that never changes is made once), per layer tsfm_rope_append_tree and
 * tsfm_tree_attention, then tsfm_verify_tree on the target's probabilities at all nodes and tsfm_cache_commit, which
 * moves the accepted nodes' keys and values to the front.  New tokens lie in slots len[b] + m whatever the tree.
 * shared_tree != 0: what describes the tree (parent, mask, depth) has one row for all series in place of one a series. */
#define TSFM_MAX_TREE 256       /* nodes of a tree */
#define TSFM_MAX_TOP  32        /* best tokens of tsfm_token_logprobs */

/* What nodes see, and how deep they are.
 *   parent  [B, M]; one outside -1 .. m - 1 counts as -1
 *   n_new   [B] nodes, cut to 0 .. M; NULL: M each
 *   window  0, or as given to tsfm_tree_attention: ancestors `window` levels above or more are not seen
 *   mask    [B, M, ceil(M / 64)] uint64 out: bit j % 64 of word j / 64 of node m: m sees j, itself or an ancestor
 *   depth   [B, M] out: ancestors of m
 * Nodes behind n_new get 0.  M <= TSFM_MAX_TREE. */
int tsfm_tree_init(void *stream, const int32_t *parent, const int32_t *n_new, int32_t B, int32_t M, int32_t window, uint64_t *mask, int32_t *depth);

/* tsfm_rope_append for a tree: node m has position pos[b] + depth[m] (and slot len[b] + m).  depth: [B, M] or [M]. */
int tsfm_rope_append_tree(void *stream, const tsfm_rope *rope, const tsfm_kv_pages *pages, const void *qkv, int64_t qkv_stride, void *q_out,
                          int64_t q_out_stride, const int32_t *pos, const int32_t *len, const int32_t *n_new, const int32_t *depth, int32_t shared_tree,
                          int32_t B, int32_t M, int32_t n_heads);

/* Attention of a tree over the cache, its nodes' keys and values already in it.  Node m < n_new[b] stands at len[b] + depth[m] and sees
 *   slots s < len[b] with s > len[b] + depth[m] - window or s < sinks (window 0: all of them), and
 *   slots len[b] + j, j < n_new[b], with bit j of mask[m].  (Any mask: it need not come from tsfm_tree_init.)
 *   mask     [B, M, ceil(M / 64)] or [M, ceil(M / 64)]
 *   depth    [B, M] or [M], cut to 0 .. M - 1; may be NULL with window 0
 *   max_len  the longest series in slots, new ones included: lengths are cut to it.  It sizes the grid and the workspace, not the work
 *   workspace  256-byte aligned, tsfm_tree_attention_workspace() bytes; contents do not matter.  Calls that may overlap (two streams, two
 *            graphs) need one each
 * Head layouts, rows that see nothing, hidden slots, rows behind n_new, precision, lse and status: as tsfm_paged_attention.  A series' queries behind n_new may
 * hold anything.
 * M <= TSFM_MAX_TREE. */
int tsfm_tree_attention(void *stream, const tsfm_kv_pages *pages, const void *q, int64_t q_stride, void *out, int64_t out_stride,
                        const int32_t *len, const int32_t *n_new, const uint64_t *mask, const int32_t *depth, int32_t shared_tree, int32_t B,
                        int32_t M, int32_t n_heads, float scale, int32_t window, int32_t sinks, int32_t max_len, float *lse, void *workspace,
                        size_t workspace_bytes);

/* Attention of new tokens one behind the other, their keys and values already in the cache, within a sliding window that keeps the first
 * slots visible: token m < n_new[b] sees slots s <= len[b] + m with s > len[b] + m - window or s < sinks (window 0: all of them).
 * One token or a prompt: a token's rows read what they see.  M n_heads / n_kv_heads at most 65535.  Otherwise as
 * tsfm_tree_attention, with its workspace. */
int tsfm_window_attention(void *stream, const tsfm_kv_pages *pages, const void *q, int64_t q_stride, void *out, int64_t out_stride,
                          const int32_t *len, const int32_t *n_new, int32_t B, int32_t M, int32_t n_heads, float scale, int32_t window,
                          int32_t sinks, int32_t max_len, float *lse, void *workspace, size_t workspace_bytes);

/* Bytes of workspace for either call (host arithmetic only; of `pages` the shapes and the dtype count).  0 on invalid arguments. */
size_t tsfm_tree_attention_workspace(const tsfm_kv_pages *pages, int32_t B, int32_t M, int32_t n_heads, int32_t max_len);

/* Log probabilities of rows of logits: x = scale * logit, lse = log sum e^x, p = e^(x - lse).  A draft grows its tree from the
 * best tokens; a server returns what was likely and how sure the model was.
 *   logits   [rows] rows of V elements of dtype (TSFM_F32, TSFM_BF16), `stride` elements apart, at any alignment of an element
 *   tokens   [rows, n_tokens] int32; NULL with n_tokens 0
 *   logprob  [rows, n_tokens] out: x - lse of those tokens (outside [0, V): -inf)
 *   lse      [rows] out, nullable;  entropy [rows] out, nullable: lse - sum p x, with p x = 0 where p is 0
 *   top_ids  [rows, n_top] out: the n_top tokens with the largest logits, largest first, among equals the lower token first (NaN lies
 *            below -inf); -1 behind the V-th.  top_logprob: their x - lse; -inf behind the V-th
 * Sums are fp32.  Logits of -inf are tokens that cannot be; a row of them has lse and log probabilities -inf and entropy 0.  NaN or +inf in a
 * row make its lse, entropy and log probabilities NaN.  scale > 0; n_top <= TSFM_MAX_TOP; V <= 2^30. */
int tsfm_token_logprobs(void *stream, const void *logits, int64_t stride, int32_t dtype, int32_t rows, int32_t V, float scale, const int32_t *tokens,
                        int32_t n_tokens, float *logprob, float *lse, float *entropy, int32_t n_top, int32_t *top_ids, float *top_logprob);

/* Verification of a tree: from node 0 on, the children of the node reached are tried in order of their numbers; the first accepted one is
 * reached next, and where none is, a token is drawn.  At node c, with r = p_c, Z = 1 and C = 0 at first, child j (token x) is accepted if
 *     u_j q_c(x) Z < r(x);     else C += Z, r = max(p_c - C q_c, 0), Z = sum r
 * in fp64: children drawn independently from q_c leave the committed tokens distributed as the target's.  q NULL: the draft's best
 * tokens, q_c(x) is 1 at the child tried and 0 elsewhere: r loses the rejected tokens, Z their p.  The token behind the path is drawn
 * from r as tsfm_verify_tokens draws (and from p_c where r is 0 everywhere).  Entries of p and q that are negative or not finite count as 0,
 * uniforms are cut to [0, 1 - 2^-24], a token outside [0, V) is rejected, a node that node 0 does not lead to is not reached.
 *   tokens, parent  [B, M] (parent: [M] with shared_tree; outside -1 .. m - 1 counts as -1); tokens[b][0] is not read as a proposal
 *   p       [B, M] rows of V fp32, p_stride elements apart: the target's probabilities behind each node
 *   q       [B, M] rows of V fp32, q_stride apart: the draft's; nullable
 *   u       [B, M + 1] fp32 uniforms, one a node and the last for the draw; NULL: the Philox uniforms of tsfm_accept_round, counter
 *           (series0 + b, round_idx, node, 0), key = seed
 *   n_new   [B] nodes, cut to 0 .. M; NULL: M each
 *   out     [B, M] int32: the n accepted tokens and the drawn one, -1 behind them (the drawn one is -1 too where p has no positive entry)
 *   path    [B, M] int32: node 0 and the n accepted nodes, -1 behind them: what tsfm_cache_commit takes
 *   n_accept [B] int32 out: n
 *   len, len_out  [B] int32, both or neither: len_out = len + n + 1; may be the same
 * A series without nodes commits nothing: out and path -1, n 0, len_out = len.  M <= TSFM_MAX_TREE, V <= 2^30.  Outputs overlap no input. */
int tsfm_verify_tree(void *stream, const int32_t *tokens, const int32_t *parent, int32_t shared_tree, const float *p, int64_t p_stride, const float *q,
                     int64_t q_stride, int32_t B, int32_t M, int32_t V, const float *u, uint64_t seed, int32_t round_idx, int32_t series0,
                     const int32_t *n_new, const int32_t *len, int32_t *out, int32_t *path, int32_t *n_accept, int32_t *len_out);

/* The accepted path's keys and values to the front: slot len[b] + path[b][i] goes to slot len[b] + i, in place, for every i up to the first
 * entry that is negative, M or more, or not above the one before.
 *   path      [B, M] int32, as tsfm_verify_tree writes it
 *   len       [B] slots before the tree (not tsfm_verify_tree's len_out)
 *   n_layers  pools that lie layer_stride elements apart, k and v alike, with one table for all (1: pages as they are)
 * Slots outside the capacity and pages outside the pool are left alone and set bits of *status.  The pages belong to one series only.
 * M <= TSFM_MAX_TREE. */
int tsfm_cache_commit(void *stream, const tsfm_kv_pages *pages, const int32_t *path, const int32_t *len, int32_t B, int32_t M, int32_t n_layers,
                      int64_t layer_stride);

/* Bounds-checking mode only (TSFM_EXEC_CHECK_BOUNDS): *n_regions (nullable) receives the number of
 * guard regions of the handle.  region >= 0 additionally overwrites (damage != 0) or restores
 * (damage == 0) one byte of that guard region -- a write inside the library's own allocation --
 * so that a test can see the checker report it.  region < 0: query only. */
int tsfm_spec_debug_guard(tsfm_spec *h, int32_t region, int32_t damage, int32_t *n_regions);

/* Per-launch timing, for roofline accounting.  While enabled, every kernel launch of the handle
 * is bracketed by two CUDA events on the handle's stream (this perturbs end-to-end time: do not
 * quote throughput from a profiled call).  tsfm_spec_set_profiling clears the records.
 * tsfm_spec_kernel_profile synchronises and aggregates them per kernel: launches, total device
 * milliseconds, and the algorithmic bytes and flops of those launches (what the operation must
 * move / compute: operands read once, results written once).  out: host array of `cap` entries;
 * *n receives the number of kernels with at least one launch. */
typedef struct {
  char    name[24];
  int64_t launches;
  double  ms_total;
  double  bytes;
  double  flops;
} tsfm_kernel_stat;
int tsfm_spec_set_profiling(tsfm_spec *h, int32_t enable);
int tsfm_spec_kernel_profile(tsfm_spec *h, int32_t cap, int32_t *n, tsfm_kernel_stat *out);

/* Block-size advice from measured quantities (host arithmetic only).  alpha = conditional
 * acceptance rate, c = draft step cost and v = verification pass cost in units of one target step.
 * Expected yield E[L_K] = sum_{j=0..K} alpha^j (Eq. 7), predicted speedup S(K) = E[L_K] / (c K + v)
 * (Eq. 8).  Steps K up from 1 while the marginal-gain condition alpha^(K+1) (c K + v) >= c E[L_K]
 * of the block-size proposition holds (it is equivalent to S(K+1) >= S(K)) and returns the K reached,
 * at most max_K; *speedup (nullable) receives S at that K.  Returns 0 on invalid arguments
 * (alpha outside [0, 1], c <= 0, v <= 0, max_K < 1). */
int32_t tsfm_advise_block_size(double alpha, double c, double v, int32_t max_K, double *speedup);

int tsfm_spec_destroy(tsfm_spec *h);

/* Number of kernels this library has launched in this process (all handles, all streams).  The
 * rounds of a graph-mode forecast count their launches on the device: the call waits for the
 * streams of all live handles to read those counters. */
int64_t tsfm_launch_count(void);

const char *tsfm_strerror(int code);
/* Text of the last CUDA error that produced TSFM_ERR_CUDA on this thread ("" if none). */
const char *tsfm_last_cuda_error(void);

#ifdef __cplusplus
}
#endif
#endif /* TSFM_H_ */
