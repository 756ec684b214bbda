// C entry points for trees of drafted tokens, windows with first slots, and log probabilities (the section of that name in
// include/tsfm.h): argument checks, launch shapes.
#pragma once
#include "attn_tree_tc.cuh"
#include "token_logprobs.cuh"
#include "tree.cuh"
#include "verify_tree.cuh"

namespace {

static_assert(TREE_MAX == TSFM_MAX_TREE && LP_MAX_TOP == TSFM_MAX_TOP, "as include/tsfm.h says");

// Whether the rows of a key head go to tree_attn_tc_kernel, as far as shapes say: heads of 64 from 33 rows on, heads of 128 from 17.  (It takes 128 at a time, the
// other kernel 8, 16 or 32; us there and in the other.  64 x 20 heads of 64, 346 slots: 17 rows 85 and 54, 30 rows 87 and 60, 33 rows 86 and 111.  16 x 8 heads
// of 128, 4096 slots: 16 rows 73 and 59, 17 rows 73 and 93, 64 rows 78 and 169; 64 x 8 heads, 2048 slots, 20 rows: 136 and 181; 4 x 8 heads, 32 rows: 32 and 27.)
constexpr int TREE_TC_MIN_ROWS_64 = 33, TREE_TC_MIN_ROWS_128 = 17;
bool tree_on_tc(const tsfm_kv_pages *p, int M, int n_heads) {
  return p->dtype == TSFM_BF16 && p->d_head >= 64 && p->page_size >= 8 &&
         (long long)M * (n_heads / p->n_kv_heads) >= (p->d_head == 64 ? TREE_TC_MIN_ROWS_64 : TREE_TC_MIN_ROWS_128);
}
// Plan of either kernel; windows: each chunk of rows has a window of its own; pl->bytes: what both would need (a pool's strides, which say whether TMA can read it, are not known here).
int tree_plan(PagedPlan *pl, PagedPlan *tc, bool windows, const tsfm_kv_pages *p, int B, int M, int n_heads, int max_len) {
  if (int rc = paged_plan(pl, p, B, M, n_heads, max_len, false)) return rc;
  *tc = *pl;
  if (!tree_on_tc(p, M, n_heads)) return TSFM_OK;
  const long long R = (long long)M * (n_heads / p->n_kv_heads), pairs = (long long)B * p->n_kv_heads;
  // A CTA takes 256 rows beside one another, which share the slots that they read, where there are more than 128; but 257 to 384 rows are three times 128 and a
  // unit of 256 would do half of its work for none.  (32 series of 2048 slots, 8 key heads of 128, us with 256 and with 128: 244 rows 148 and 164, 320 rows 245
  // and 214, 400 rows 249 and 281, 640 rows 378 and 386, 1020 rows 502 and 602; a chain of these 527 and 574, one chain of 8192 tokens, 4 heads a group, 798 and
  // 839.)  Chunks of a chain that have each a window of their own stay at 128: more rows make it longer, by a tile of its ten in prompts of any length (4 prompts
  // of up to 4096 tokens, window 1024: 567 and 539; window 512 391 and 378; window 4096 1182 and 1254; lengths of whole blocks, window 1024: 496 and 511).
  tc->rows = R <= 128 || windows || (R > 256 && R <= 384) ? 128 : 256;
  tc->chunks = (int)((R + tc->rows - 1) / tc->rows);
  tc->grid = (int)std::min<long long>(pairs * tc->chunks * ((max_len + 2 * PA_TILE - 1) / (2 * PA_TILE) + 1), 2 * kSms * 128 / tc->rows);
  size_t at = align256(sizeof(PagedMeta) * tc->grid);
  tc->part_ml = at;
  at = align256(at + sizeof(float2) * 2 * tc->grid * tc->rows);
  tc->part_o = at;
  tc->bytes = align256(at + sizeof(float) * 2 * tc->grid * tc->rows * p->d_head);
  tc->bytes = pl->bytes = std::max(pl->bytes, tc->bytes);
  return TSFM_OK;
}

// Map of the queries: {element, head, token}, boxes of a group's heads x the tokens that make 128 rows.
bool query_map(CUtensorMap *q, const PagedAttnArgs &a, int D) {
  if (128 % a.group || a.q_stride * 2 >= 1ll << 40) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)a.n_heads, (cuuint64_t)a.B * a.M}, strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)a.q_stride * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)a.group, (cuuint32_t)(128 / a.group)}, one[3] = {1, 1, 1};
  return tensor_map_encoder()(q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(a.q), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
template <typename C> cudaError_t launch_tree_tc(cudaStream_t s, const PagedAttnArgs &a, const PagedPlan &pl, const CUtensorMap &k, const CUtensorMap &v) {
  if (cudaError_t e = cudaFuncSetAttribute(tree_attn_tc_kernel<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES)) return e;
  CUtensorMap q{};
  const int q_tma = query_map(&q, a, C::D);
  tree_attn_tc_kernel<C><<<pl.grid, C::THREADS, C::SMEM_BYTES, s>>>(a, k, v, q, q_tma);
  if (cudaError_t e = cudaGetLastError()) return e;
  LAUNCHED();
  return join_paged<bf16, C::D, true>(s, a, pl);
}

// tsfm_tree_attention (mask or a chain) and tsfm_window_attention
int tree_attention(void *stream, const tsfm_kv_pages *pages, const void *q, int64_t q_stride, void *out, int64_t out_stride, const int32_t *len,
                   const int32_t *n_new, const uint64_t *mask, const int32_t *depth, bool shared, int32_t B, int32_t M, int32_t n_heads, float scale,
                   int32_t window, int32_t sinks, int32_t max_len, float *lse, void *workspace, size_t workspace_bytes) {
  if (!q || !out || !len || !workspace || window < 0 || sinks < 0 || !std::isfinite(scale * kLog2E)) return TSFM_ERR_ARG;
  PagedPlan pl, tc;
  if (int rc = tree_plan(&pl, &tc, !mask && window, pages, B, M, n_heads, max_len)) return rc;
  PagedAttnArgs a{};
  CUtensorMap k{}, v{};
  if (tree_on_tc(pages, M, n_heads)) {
    if (int rc = pages_init(&a.pg, pages)) return rc;
    if (paged_maps(&k, &v, a.pg, pages->d_head, 2)) pl = tc;
  }
  if (int rc = paged_args(&a, pl, pages, q, q_stride, out, out_stride, len, n_new, B, M, n_heads, scale, window, max_len, lse, workspace, workspace_bytes)) return rc;
  a.causal = 1;
  a.mask = (const unsigned long long *)mask;
  a.depth = depth;
  a.words = (M + 63) / 64;
  a.mask_series = shared ? 0 : (long long)M * a.words;
  a.depth_series = shared ? 0 : M;
  a.sinks = window ? sinks : 0;
  cudaStream_t s = (cudaStream_t)stream;
  const int D = pages->d_head;
  cudaError_t err;
  if (pl.rows == 128)
    err = D == 64 ? launch_tree_tc<TreeTc<64, 1>>(s, a, pl, k, v) : launch_tree_tc<TreeTc<128, 1>>(s, a, pl, k, v);
  else if (pl.rows == 256)
    err = D == 64 ? launch_tree_tc<TreeTc<64, 2>>(s, a, pl, k, v) : launch_tree_tc<TreeTc<128, 2>>(s, a, pl, k, v);
  else if (pages->dtype == TSFM_BF16)
    err = D == 32 ? launch_paged<bf16, 32, true>(s, a, pl) : D == 64 ? launch_paged<bf16, 64, true>(s, a, pl) : launch_paged<bf16, 128, true>(s, a, pl);
  else
    err = D == 32 ? launch_paged<float, 32, true>(s, a, pl) : D == 64 ? launch_paged<float, 64, true>(s, a, pl) : launch_paged<float, 128, true>(s, a, pl);
  CU_TRY(err);
  return TSFM_OK;
}

}  // namespace

extern "C" {

int tsfm_tree_init(void *stream, const int32_t *parent, const int32_t *n_new, int32_t B, int32_t M, int32_t window, uint64_t *mask, int32_t *depth) {
  if (!parent || !mask || !depth || B < 1 || M < 1 || window < 0) return TSFM_ERR_ARG;
  if (M > TREE_MAX) return TSFM_ERR_SHAPE;
  tree_init_kernel<<<B, TREE_MAX, 0, (cudaStream_t)stream>>>(parent, n_new, M, (M + 63) / 64, window, (unsigned long long *)mask, depth);
  CU_TRY(cudaGetLastError());
  LAUNCHED();
  return TSFM_OK;
}

int tsfm_rope_append_tree(void *stream, const tsfm_rope *rope, const tsfm_kv_pages *pages, const void *qkv, int64_t qkv_stride, void *q_out,
                          int64_t q_out_stride, const int32_t *pos, const int32_t *len, const int32_t *n_new, const int32_t *depth, int32_t shared_tree,
                          int32_t B, int32_t M, int32_t n_heads) {
  if (!depth) return TSFM_ERR_ARG;
  return rope_append(stream, rope, pages, qkv, qkv_stride, q_out, q_out_stride, pos, len, n_new, depth, shared_tree != 0, B, M, n_heads);
}

size_t tsfm_tree_attention_workspace(const tsfm_kv_pages *pages, int32_t B, int32_t M, int32_t n_heads, int32_t max_len) {
  PagedPlan pl, with_windows, tc;
  if (tree_plan(&pl, &tc, false, pages, B, M, n_heads, max_len) || tree_plan(&with_windows, &tc, true, pages, B, M, n_heads, max_len)) return 0;
  return std::max(pl.bytes, with_windows.bytes);
}

int tsfm_tree_attention(void *stream, const tsfm_kv_pages *pages, const void *q, int64_t q_stride, void *out, int64_t out_stride,
                        const int32_t *len, const int32_t *n_new, const uint64_t *mask, const int32_t *depth, int32_t shared_tree, int32_t B,
                        int32_t M, int32_t n_heads, float scale, int32_t window, int32_t sinks, int32_t max_len, float *lse, void *workspace,
                        size_t workspace_bytes) {
  if (!mask || (window && !depth)) return TSFM_ERR_ARG;
  if (M > TREE_MAX) return TSFM_ERR_SHAPE;
  return tree_attention(stream, pages, q, q_stride, out, out_stride, len, n_new, mask, depth, shared_tree != 0, B, M, n_heads, scale, window, sinks, max_len,
                        lse, workspace, workspace_bytes);
}

int tsfm_window_attention(void *stream, const tsfm_kv_pages *pages, const void *q, int64_t q_stride, void *out, int64_t out_stride,
                          const int32_t *len, const int32_t *n_new, int32_t B, int32_t M, int32_t n_heads, float scale, int32_t window,
                          int32_t sinks, int32_t max_len, float *lse, void *workspace, size_t workspace_bytes) {
  return tree_attention(stream, pages, q, q_stride, out, out_stride, len, n_new, nullptr, nullptr, false, B, M, n_heads, scale, window, sinks, max_len, lse,
                        workspace, workspace_bytes);
}

int tsfm_token_logprobs(void *stream, const void *logits, int64_t stride, int32_t dtype, int32_t rows, int32_t V, float scale, const int32_t *tokens,
                        int32_t n_tokens, float *logprob, float *lse, float *entropy, int32_t n_top, int32_t *top_ids, float *top_logprob) {
  if (!logits || (dtype != TSFM_F32 && dtype != TSFM_BF16) || rows < 1 || V < 1 || n_tokens < 0 || n_top < 0) return TSFM_ERR_ARG;
  if (!(scale > 0) || !std::isfinite(scale * kLog2E) || stride < V) return TSFM_ERR_ARG;
  if ((n_tokens && (!tokens || !logprob)) || (n_top && (!top_ids || !top_logprob))) return TSFM_ERR_ARG;
  const int e = (int)elt_bytes(dtype);
  if (n_top > LP_MAX_TOP || V > kMaxSlots || stride > (INT64_MAX >> 4) || (uintptr_t)logits % e) return TSFM_ERR_SHAPE;
  LogprobArgs a{};
  a.x = logits;
  a.stride = stride;
  a.V = V;
  a.scale = scale;
  a.scale2 = scale * kLog2E;
  a.tokens = tokens;
  a.n_tokens = n_tokens;
  a.logprob = logprob;
  a.lse = lse;
  a.entropy = entropy;
  a.n_top = n_top;
  a.ids = top_ids;
  a.best = top_logprob;
  // few rows are shared by CTAs, of 16 entries for each thread at least
  int cluster = 1;
  while (cluster < LP_MAX_CLUSTER && 2ll * rows * cluster <= 4 * kSms && V > (long long)cluster * LP_THREADS * 16) cluster *= 2;
  if ((long long)rows * cluster > kMaxGridX) return TSFM_ERR_SHAPE;
  auto launch = [&](auto kernel) { return launch_cluster((cudaStream_t)stream, (unsigned)(rows * cluster), LP_THREADS, 0, cluster, kernel, a); };
  CU_TRY(dtype == TSFM_BF16 ? launch(token_logprobs_kernel<bf16>) : launch(token_logprobs_kernel<float>));
  LAUNCHED();
  return TSFM_OK;
}

int tsfm_verify_tree(void *stream, const int32_t *tokens, const int32_t *parent, int32_t shared_tree, const float *p, int64_t p_stride, const float *q,
                     int64_t q_stride, int32_t B, int32_t M, int32_t V, const float *u, uint64_t seed, int32_t round_idx, int32_t series0,
                     const int32_t *n_new, const int32_t *len, int32_t *out, int32_t *path, int32_t *n_accept, int32_t *len_out) {
  if (!tokens || !parent || !p || !out || !path || !n_accept || B < 1 || M < 1 || V < 1 || !len != !len_out) return TSFM_ERR_ARG;
  if (p_stride < V || (q && q_stride < V)) return TSFM_ERR_ARG;
  if (M > TREE_MAX || V > kMaxSlots) return TSFM_ERR_SHAPE;
  VerifyTreeArgs a{};
  a.tokens = tokens;
  a.parent = parent;
  a.parent_series = shared_tree ? 0 : M;
  a.p = p;
  a.q = q;
  a.p_stride = p_stride;
  a.q_stride = q_stride;
  a.M = M;
  a.V = V;
  a.u = u;
  a.key = make_uint2((uint32_t)(seed & 0xffffffffu), (uint32_t)(seed >> 32));
  a.round_idx = round_idx;
  a.series0 = series0;
  a.n_new = n_new;
  a.len = len;
  a.out = out;
  a.path = path;
  a.n_accept = n_accept;
  a.len_out = len_out;
  // as tsfm_verify_tokens
  int cluster = 1, warps = 4;
  while (cluster < VERIFY_MAX_CLUSTER && 2ll * B * cluster <= 8 * kSms && V > cluster * 4096) cluster *= 2;
  while (warps < VERIFY_MAX_WARPS && 2ll * B * cluster * warps <= 32 * kSms && V > cluster * warps * 512) warps *= 2;
  if ((long long)B * cluster > kMaxGridX) return TSFM_ERR_SHAPE;
  CU_TRY(launch_cluster((cudaStream_t)stream, (unsigned)(B * cluster), 32 * warps, 0, cluster, verify_tree_kernel, a));
  LAUNCHED();
  return TSFM_OK;
}

int tsfm_cache_commit(void *stream, const tsfm_kv_pages *pages, const int32_t *path, const int32_t *len, int32_t B, int32_t M, int32_t n_layers,
                      int64_t layer_stride) {
  if (!path || !len || B < 1 || M < 1 || n_layers < 1) return TSFM_ERR_ARG;
  CommitArgs a{};
  if (int rc = pages_init(&a.pg, pages)) return rc;
  const int e = (int)elt_bytes(pages->dtype);
  if (M > TREE_MAX || (n_layers > 1 && !stride_ok(layer_stride, pages->d_head, e))) return TSFM_ERR_SHAPE;
  a.path = path;
  a.len = len;
  a.layer_stride = n_layers > 1 ? layer_stride * e : 0;
  a.B = B;
  a.M = M;
  a.n_layers = n_layers;
  a.vecs = pages->d_head * e / 16;
  const long long items = (long long)n_layers * pages->n_kv_heads * 2 * a.vecs;
  a.blocks = (int)std::min<long long>((items + COMMIT_THREADS - 1) / COMMIT_THREADS, std::max<long long>(1, 16 * kSms / B));
  if ((long long)B * a.blocks > kMaxGridX) return TSFM_ERR_SHAPE;
  cache_commit_kernel<<<B * a.blocks, COMMIT_THREADS, 0, (cudaStream_t)stream>>>(a);
  CU_TRY(cudaGetLastError());
  LAUNCHED();
  return TSFM_OK;
}

}  // extern "C"
