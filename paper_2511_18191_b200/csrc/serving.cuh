// C entry points for serving over a cache of pages (the section of that name in include/tsfm.h): argument checks, launch
// shapes, workspace layout.
#pragma once
#include "attn_paged.cuh"
#include "attn_paged_f32.cuh"
#include "attn_paged_mma.cuh"
#include "cache_evict.cuh"
#include "pages.cuh"
#include "rope_append.cuh"
#include "verify_tokens.cuh"

namespace {

constexpr int kSms = 148;
constexpr long long kMaxSlots = 1 << 30;           // of a series: slot arithmetic is 32-bit
constexpr long long kMaxGridX = 0x7fffffff;
constexpr long long kMaxScores = 1ll << 48;        // of a workspace: far above any memory, far below what its size in bytes can say

// Limit of a wait for a tile, and the tile of a CTA from which on it runs out (tsfm_debug_tile_wait).
unsigned long long g_tile_wait_ns = TC_WAIT_NS;
int g_tile_miss_from = INT_MAX;

constexpr float kLog2E = 1.4426950408889634f;      // scores are kept in base 2
bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
bool stride_ok(int64_t stride, int64_t least, int e) { return stride >= least && stride <= (INT64_MAX >> 4) && stride * e % 16 == 0; }

int pages_shape(const tsfm_kv_pages *p) {
  if (!p || (p->dtype != TSFM_F32 && p->dtype != TSFM_BF16) || p->n_kv_heads < 1) return TSFM_ERR_ARG;
  if (p->d_head != 32 && p->d_head != 64 && p->d_head != 128) return TSFM_ERR_SHAPE;
  return TSFM_OK;
}

int pages_init(PagesDev *d, const tsfm_kv_pages *p) {
  if (int rc = pages_shape(p)) return rc;
  if (!p->k || !p->v || !p->table || p->max_pages < 1 || p->table_stride < p->max_pages || p->n_pages < 1 || p->page_size < 1)
    return TSFM_ERR_ARG;
  const int e = (int)elt_bytes(p->dtype);
  if (p->page_size > 65536 || (p->page_size & (p->page_size - 1))) return TSFM_ERR_SHAPE;
  if (!aligned16(p->k) || !aligned16(p->v) || !stride_ok(p->page_stride, p->d_head, e) || !stride_ok(p->head_stride, p->d_head, e) ||
      !stride_ok(p->slot_stride, p->d_head, e))
    return TSFM_ERR_SHAPE;
  d->k = (char *)p->k;
  d->v = (char *)p->v;
  d->page_stride = p->page_stride * e;
  d->head_stride = p->head_stride * e;
  d->slot_stride = p->slot_stride * e;
  d->table = p->table;
  d->table_stride = p->table_stride;
  d->n_pages = p->n_pages;
  for (d->page_log = 0; 1 << d->page_log < p->page_size;) ++d->page_log;
  d->n_kv_heads = p->n_kv_heads;
  d->capacity = (int)std::min<long long>(kMaxSlots, (long long)p->max_pages * p->page_size);
  d->status = p->status;
  return TSFM_OK;
}

template <typename... KArgs, typename... Args>
cudaError_t launch_after(cudaStream_t s, dim3 grid, int threads, void (*kernel)(KArgs...), const Args &...args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

template <typename... KArgs, typename... Args>
cudaError_t launch_cluster(cudaStream_t s, unsigned grid, int threads, size_t smem, int cluster, void (*kernel)(KArgs...), const Args &...args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

// The workspace of tsfm_paged_attention: rows of a unit, CTAs, and where the parts of it begin.
struct PagedPlan {
  int rows, chunks, grid;
  size_t part_ml, part_o, lse2, scores, bytes;
  long long score_stride;
};
// The kernel of `rows` rows: f gets its configuration.
template <int D, bool TREE, typename F> auto paged_variant(bf16, int rows, F f) {
  return rows == 8 ? f(PagedMma<D, 1, 1, TREE>()) : rows == 16 ? f(PagedMma<D, 2, 1, TREE>()) : f(PagedMma<D, 2, 2, TREE>());
}
template <int D, bool TREE, typename F> auto paged_variant(float, int rows, F f) {
  return rows == 1   ? f(PagedF32<D, 1, 1, TREE>())
         : rows == 2 ? f(PagedF32<D, 2, 1, TREE>())
         : rows == 4 ? f(PagedF32<D, 4, 1, TREE>())
         : rows == 8 ? f(PagedF32<D, 4, 2, TREE>())
                     : f(PagedF32<D, 4, 4, TREE>());
}
template <typename T> int paged_ctas(int D, int rows) {
  auto ctas = [](auto c) { return decltype(c)::CTAS; };
  return D == 32 ? paged_variant<32, false>(T(), rows, ctas) : D == 64 ? paged_variant<64, false>(T(), rows, ctas) : paged_variant<128, false>(T(), rows, ctas);
}
int paged_plan(PagedPlan *pl, const tsfm_kv_pages *p, int B, int M, int n_heads, int max_len, bool weights) {
  if (int rc = pages_shape(p)) return rc;
  if (B < 1 || M < 1 || n_heads < 1 || max_len < 1) return TSFM_ERR_ARG;
  if (n_heads % p->n_kv_heads) return TSFM_ERR_SHAPE;
  const long long R = (long long)M * (n_heads / p->n_kv_heads), pairs = (long long)B * p->n_kv_heads;
  if (max_len > kMaxSlots || R > 65535 || pairs > kMaxGridX || (long long)B * M > kMaxGridX) return TSFM_ERR_SHAPE;
  const bool half = p->dtype == TSFM_BF16;
  pl->rows = half ? (R <= 8 ? 8 : R <= 16 ? 16 : 32) : R <= 2 ? (int)R : R <= 4 ? 4 : R <= 8 ? 8 : 16;
  const int ctas = half ? paged_ctas<bf16>(p->d_head, pl->rows) : paged_ctas<float>(p->d_head, pl->rows);
  pl->chunks = (int)((R + pl->rows - 1) / pl->rows);
  if (pairs * pl->chunks > kMaxGridX) return TSFM_ERR_SHAPE;
  const long long tiles = pairs * pl->chunks * ((max_len + PA_TILE - 1) / PA_TILE);
  pl->grid = (int)std::min<long long>(tiles, (long long)ctas * kSms);
  size_t at = align256(sizeof(PagedMeta) * pl->grid);
  auto take = [&](size_t bytes) { const size_t o = at; at = align256(at + bytes); return o; };
  pl->part_ml = take(sizeof(float2) * 2 * pl->grid * pl->rows);
  pl->part_o = take(sizeof(float) * 2 * pl->grid * pl->rows * p->d_head);
  pl->score_stride = ((long long)max_len + 31) / 32 * 32;
  if (weights && pairs * R > kMaxScores / pl->score_stride) return TSFM_ERR_SHAPE;
  pl->lse2 = weights ? take(sizeof(float) * pairs * R) : 0;
  pl->scores = weights ? take(sizeof(float) * pairs * R * pl->score_stride) : 0;
  pl->bytes = at;
  return TSFM_OK;
}

// What both attention calls say alike: the pages, the queries and outputs, the workspace.
int paged_args(PagedAttnArgs *a, const PagedPlan &pl, const tsfm_kv_pages *pages, const void *q, int64_t q_stride, void *out, int64_t out_stride,
               const int32_t *len, const int32_t *n_new, int B, int M, int n_heads, float scale, int window, int max_len, float *lse,
               void *workspace, size_t workspace_bytes) {
  if (int rc = pages_init(&a->pg, pages)) return rc;
  const int e = (int)elt_bytes(pages->dtype);
  const int64_t row = (int64_t)n_heads * pages->d_head;
  if (!aligned16(q) || !aligned16(out) || !stride_ok(q_stride, row, e) || !stride_ok(out_stride, row, e)) return TSFM_ERR_SHAPE;
  if ((uintptr_t)workspace & 255 || workspace_bytes < pl.bytes) return TSFM_ERR_SHAPE;
  a->pg.capacity = std::min(a->pg.capacity, max_len);
  a->q = q;
  a->out = out;
  a->q_stride = q_stride;
  a->out_stride = out_stride;
  a->len = len;
  a->n_new = n_new;
  a->B = B;
  a->M = M;
  a->n_heads = n_heads;
  a->group = n_heads / pages->n_kv_heads;
  a->group_magic = (uint32_t)(((1ull << 32) + a->group - 1) / a->group);
  a->scale2 = scale * kLog2E;
  a->window = window;
  a->lse = lse;
  a->chunks = pl.chunks;
  a->units = pages->n_kv_heads * pl.chunks;
  char *ws = (char *)workspace;
  a->meta = (PagedMeta *)ws;
  a->part_ml = (float2 *)(ws + pl.part_ml);
  a->part_o = (float *)(ws + pl.part_o);
  a->wait_ns = g_tile_wait_ns;
  a->miss_from = g_tile_miss_from;
  return TSFM_OK;
}

// The driver's encoder of maps for TMA, or NULL.
PFN_encodeTiled tensor_map_encoder() {
  static const PFN_encodeTiled encode = [] {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult res{};
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &res) != cudaSuccess || res != cudaDriverEntryPointSuccess) fn = nullptr;
    return (PFN_encodeTiled)fn;
  }();
  return encode;
}
// Maps of the pool for TMA: {element, slot, head, page}, boxes of 128 (64) bytes and up to 64 slots of a page.  False where the driver
// has no encoder or refuses the pool's strides.
bool paged_maps(CUtensorMap *k, CUtensorMap *v, const PagesDev &pg, int D, int e) {
  const PFN_encodeTiled encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint32_t page = 1u << pg.page_log;
  const cuuint64_t dims[4] = {(cuuint64_t)D, page, (cuuint64_t)pg.n_kv_heads, (cuuint64_t)pg.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)pg.slot_stride, (cuuint64_t)pg.head_stride, (cuuint64_t)pg.page_stride};
  const cuuint32_t box[4] = {(cuuint32_t)std::min(D, 128 / e), std::min(page, 64u), 1, 1}, one[4] = {1, 1, 1, 1};
  for (int i = 0; i < 2; ++i)
    if (encode(i ? v : k, e == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, i ? pg.v : pg.k, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
               D * e == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return false;
  return true;
}

template <typename C, typename Kernel>
cudaError_t launch_paged_tiles(cudaStream_t s, const PagedAttnArgs &a, const PagedPlan &pl, const CUtensorMap &k, const CUtensorMap &v, Kernel kernel) {
  // (the attribute belongs to the device's context: set with every call, 0.2 us)
  if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES)) return e;
  kernel<<<pl.grid, C::THREADS, C::SMEM_BYTES, s>>>(a, k, v);
  return cudaGetLastError();
}

template <typename T, int D, bool TREE>
cudaError_t join_paged(cudaStream_t s, const PagedAttnArgs &a, const PagedPlan &pl) {
  // nothing to join where no series has a second tile
  if (a.pg.capacity <= PA_TILE || pl.grid == 1) return cudaSuccess;
  // blocks for a unit's rows: with many units each has few parts and a block joins eight rows at once, else a block a row
  // (64 x 20 units of 9 rows: 8.9 us with eight blocks)
  const long long R = (long long)a.M * a.group, here = std::min<long long>(pl.rows, R);
  const unsigned rows = (unsigned)((long long)a.B * a.units * 8 >= pl.grid ? (here + PA_JOIN_WARPS - 1) / PA_JOIN_WARPS : std::min(here, 8ll));
  if (cudaError_t e = launch_after(s, dim3(pl.grid, rows), 32 * PA_JOIN_WARPS, paged_join_kernel<T, D, TREE>, a, pl.rows)) return e;
  LAUNCHED();
  return cudaSuccess;
}

template <typename T, int D, bool TREE>
cudaError_t launch_paged(cudaStream_t s, const PagedAttnArgs &a, const PagedPlan &pl) {
  CUtensorMap k{}, v{};
  const bool tma = a.pg.page_log >= 3 && paged_maps(&k, &v, a.pg, D, (int)sizeof(T));
  const cudaError_t err = paged_variant<D, TREE>(T(), pl.rows, [&](auto c) {
    using C = decltype(c);
    if constexpr (sizeof(T) == 2)
      return tma ? launch_paged_tiles<C>(s, a, pl, k, v, paged_attn_mma_kernel<C, true>) : launch_paged_tiles<C>(s, a, pl, k, v, paged_attn_mma_kernel<C, false>);
    else
      return tma ? launch_paged_tiles<C>(s, a, pl, k, v, paged_attn_f32_kernel<C, true>) : launch_paged_tiles<C>(s, a, pl, k, v, paged_attn_f32_kernel<C, false>);
  });
  if (err) return err;
  LAUNCHED();
  if (cudaError_t e = join_paged<T, D, TREE>(s, a, pl)) return e;
  if (a.w_out) {
    const long long chunks = (a.pg.capacity + 511ll) / 512;
    if (cudaError_t e = launch_after(s, dim3((unsigned)(a.B * a.pg.n_kv_heads), (unsigned)std::min(chunks, 4096ll)), 128, paged_weights_kernel, a)) return e;
    LAUNCHED();
  }
  return cudaSuccess;
}

// depth NULL: the new tokens stand one behind the other.
int rope_append(void *stream, const tsfm_rope *rope, const tsfm_kv_pages *pages, const void *qkv, int64_t qkv_stride, void *q_out, int64_t q_out_stride,
                const int32_t *pos, const int32_t *len, const int32_t *n_new, const int32_t *depth, bool shared, int32_t B, int32_t M, int32_t n_heads) {
  if (!rope || !qkv || !len || B < 1 || M < 1 || n_heads < 0 || (q_out && n_heads < 1)) return TSFM_ERR_ARG;
  if ((rope->layout != TSFM_ROPE_HALF && rope->layout != TSFM_ROPE_INTERLEAVED) || rope->rot_dim < 0 || rope->rot_dim % 2) return TSFM_ERR_ARG;
  RopeAppendArgs a{};
  if (int rc = pages_init(&a.pg, pages)) return rc;
  const int D = pages->d_head, e = (int)elt_bytes(pages->dtype);
  const int64_t row = ((int64_t)n_heads + 2ll * pages->n_kv_heads) * D;
  if (rope->rot_dim > D || (int64_t)B * M > kMaxGridX || row > 1 << 30) return TSFM_ERR_SHAPE;       // (elements of a row are counted in 32 bits)
  if (!aligned16(qkv) || !stride_ok(qkv_stride, row, e)) return TSFM_ERR_SHAPE;
  if (q_out && (!aligned16(q_out) || !stride_ok(q_out_stride, (int64_t)n_heads * D, e))) return TSFM_ERR_SHAPE;
  if (q_out == qkv && q_out_stride != qkv_stride) return TSFM_ERR_ARG;
  a.qkv = qkv;
  a.q_out = q_out;
  a.qkv_stride = qkv_stride;
  a.q_stride = q_out_stride;
  a.pos = pos;
  a.len = len;
  a.n_new = n_new;
  a.depth = depth;
  a.depth_series = shared ? 0 : M;
  a.tokens = B * M;
  a.M = M;
  a.n_heads = n_heads;
  a.half = rope->layout == TSFM_ROPE_HALF;
  a.pairs = rope->rot_dim / 2;
  a.mscale = rope->mscale;
  std::memcpy(a.turn, rope->turn, sizeof a.turn);
  if (pages->dtype == TSFM_BF16) launch_rope_append<bf16>((cudaStream_t)stream, a, D);
  else launch_rope_append<float>((cudaStream_t)stream, a, D);
  CU_TRY(cudaGetLastError());
  LAUNCHED();
  return TSFM_OK;
}

}  // namespace

extern "C" {

int tsfm_rope_init(tsfm_rope *rope, int32_t layout, int32_t rot_dim, int32_t scaling, double base, double factor,
                   double original_len, double turns_lo, double turns_hi, float mscale) {
  if (!rope || (layout != TSFM_ROPE_HALF && layout != TSFM_ROPE_INTERLEAVED) || scaling < TSFM_ROPE_PLAIN || scaling > TSFM_ROPE_PARTS)
    return TSFM_ERR_ARG;
  if (rot_dim < 0 || rot_dim > 2 * ROPE_MAX_PAIRS || rot_dim % 2) return TSFM_ERR_ARG;
  if (!(base > 1) || !std::isfinite(base) || !(factor >= 1) || !std::isfinite(factor) || !std::isfinite(mscale)) return TSFM_ERR_ARG;
  if (scaling == TSFM_ROPE_BASE && rot_dim == 2) return TSFM_ERR_ARG;
  if (scaling == TSFM_ROPE_PARTS && (!(original_len > 0) || !std::isfinite(original_len) || !(turns_lo >= 0) || !(turns_hi > turns_lo) || !std::isfinite(turns_hi)))
    return TSFM_ERR_ARG;
  std::memset(rope, 0, sizeof *rope);
  rope->layout = layout;
  rope->rot_dim = rot_dim;
  rope->mscale = mscale;
  const long double two_pi = 6.283185307179586476925286766559L;
  long double b = base;
  if (scaling == TSFM_ROPE_BASE && rot_dim > 2) b *= powl(factor, rot_dim / (rot_dim - 2.0L));
  for (int i = 0; i < rot_dim / 2; ++i) {
    long double f = powl(b, -2.0L * i / rot_dim);
    if (scaling == TSFM_ROPE_LINEAR) f /= factor;
    if (scaling == TSFM_ROPE_PARTS) {
      long double g = (original_len * f / two_pi - turns_lo) / ((long double)turns_hi - turns_lo);
      g = g < 0 ? 0 : g > 1 ? 1 : g;
      f *= g + (1 - g) / factor;
    }
    rope->turn[i] = (uint64_t)(f / two_pi * 18446744073709551616.0L + 0.5L);       // f <= 1: below 2^62
  }
  return TSFM_OK;
}

int tsfm_rope_append(void *stream, const tsfm_rope *rope, const tsfm_kv_pages *pages, const void *qkv, int64_t qkv_stride,
                     void *q_out, int64_t q_out_stride, const int32_t *pos, const int32_t *len, const int32_t *n_new,
                     int32_t B, int32_t M, int32_t n_heads) {
  return rope_append(stream, rope, pages, qkv, qkv_stride, q_out, q_out_stride, pos, len, n_new, nullptr, false, B, M, n_heads);
}

size_t tsfm_paged_attention_workspace(const tsfm_kv_pages *pages, int32_t B, int32_t M, int32_t n_heads, int32_t max_len,
                                      int32_t with_weights) {
  PagedPlan pl;
  return paged_plan(&pl, pages, B, M, n_heads, max_len, with_weights != 0) ? 0 : pl.bytes;
}

int tsfm_paged_attention(void *stream, const tsfm_kv_pages *pages, const void *q, int64_t q_stride, void *out, int64_t out_stride,
                         const int32_t *len, const int32_t *n_new, int32_t B, int32_t M, int32_t n_heads, float scale,
                         int32_t causal, int32_t window, int32_t max_len, float *lse, const float *w_in, float *w_out,
                         int64_t w_stride, void *workspace, size_t workspace_bytes) {
  if (!q || !out || !len || !workspace || window < 0 || !std::isfinite(scale * kLog2E) || (w_in && !w_out)) return TSFM_ERR_ARG;
  PagedPlan pl;
  if (int rc = paged_plan(&pl, pages, B, M, n_heads, max_len, w_out != nullptr)) return rc;
  PagedAttnArgs a{};
  if (int rc = paged_args(&a, pl, pages, q, q_stride, out, out_stride, len, n_new, B, M, n_heads, scale, window, max_len, lse, workspace, workspace_bytes)) return rc;
  if (w_out && w_stride < max_len) return TSFM_ERR_SHAPE;
  const int D = pages->d_head;
  char *ws = (char *)workspace;
  a.causal = causal != 0;
  a.w_in = w_in;
  a.w_out = w_out;
  a.w_stride = w_stride;
  a.lse2 = w_out ? (float *)(ws + pl.lse2) : nullptr;
  a.scores = w_out ? (float *)(ws + pl.scores) : nullptr;
  a.score_stride = pl.score_stride;
  cudaStream_t s = (cudaStream_t)stream;
  cudaError_t err;
  if (pages->dtype == TSFM_BF16)
    err = D == 32 ? launch_paged<bf16, 32, false>(s, a, pl) : D == 64 ? launch_paged<bf16, 64, false>(s, a, pl) : launch_paged<bf16, 128, false>(s, a, pl);
  else
    err = D == 32 ? launch_paged<float, 32, false>(s, a, pl) : D == 64 ? launch_paged<float, 64, false>(s, a, pl) : launch_paged<float, 128, false>(s, a, pl);
  CU_TRY(err);
  return TSFM_OK;
}

void tsfm_debug_tile_wait(int64_t wait_us, int32_t miss_from) {
  g_tile_wait_ns = wait_us > 0 ? std::min<unsigned long long>(TC_WAIT_NS, 1000ull * (unsigned long long)std::min<int64_t>(wait_us, 1000000)) : TC_WAIT_NS;
  g_tile_miss_from = miss_from < 0 ? INT_MAX : miss_from;
}

int tsfm_cache_evict(void *stream, const tsfm_kv_pages *pages, const int32_t *dst_table, int32_t dst_stride, const int32_t *len,
                     const float *w, int64_t w_stride, int32_t B, int32_t budget, int32_t sinks, int32_t recent, int32_t max_len,
                     int32_t *kept, float *w_out, int64_t w_out_stride, int32_t *len_out) {
  if (!dst_table || !len || !w || !kept || !len_out || len == len_out || w == w_out) return TSFM_ERR_ARG;
  if (B < 1 || budget < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget || max_len < 1) return TSFM_ERR_ARG;
  EvictArgs a{};
  if (int rc = pages_init(&a.pg, pages)) return rc;
  a.pg.capacity = std::min(a.pg.capacity, max_len);
  const long long pairs = (long long)B * pages->n_kv_heads, most = std::min(budget, a.pg.capacity);
  if (pairs > kMaxGridX || w_stride < a.pg.capacity || (w_out && w_out_stride < most)) return TSFM_ERR_SHAPE;
  if ((long long)dst_stride * pages->page_size < most) return TSFM_ERR_SHAPE;
  a.dst_table = dst_table;
  a.dst_stride = dst_stride;
  a.len = len;
  a.w = w;
  a.w_stride = w_stride;
  a.w_out_stride = w_out_stride;
  a.B = B;
  a.budget = budget;
  a.sinks = sinks;
  a.recent = recent;
  a.kept = kept;
  a.w_out = w_out;
  a.len_out = len_out;
  a.vecs = pages->d_head * (int)elt_bytes(pages->dtype) / 16;
  cudaStream_t s = (cudaStream_t)stream;
  // threads, and above 16384 slots CTAs of a cluster: what the longest series' ranks need, as far as that goes
  const int threads = a.pg.capacity <= 4096 ? 256 : a.pg.capacity <= 8192 ? 512 : 1024;
  int cluster = 1;
  while (cluster < EVICT_MAX_CLUSTER && cluster * 16 * threads < a.pg.capacity && 2 * pairs * cluster <= kMaxGridX) cluster *= 2;
  auto select = [&](auto kernel, size_t smem) {
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)) return e;
    return launch_cluster(s, (unsigned)(pairs * cluster), threads, smem, cluster, kernel, a);
  };
  CU_TRY(threads == 256   ? select(evict_select_kernel<256>, sizeof(EvictShared<256>))
         : threads == 512 ? select(evict_select_kernel<512>, sizeof(EvictShared<512>))
                          : select(evict_select_kernel<1024>, sizeof(EvictShared<1024>)));
  LAUNCHED();
  // four rows a thread once that fills the SMs (32 x 8 heads of 2048: 114 us against 120 for the whole call), else two (1 x 4 of 1024:
  // 12.4 against 14.3)
  const bool many = pairs * (most * a.vecs / 1024) >= 4 * kSms;
  const long long rows = 256 / a.vecs * (many ? 4 : 2), chunks = (most + rows - 1) / rows;
  const dim3 grid((unsigned)pairs, (unsigned)std::min(chunks, 65535ll));
  CU_TRY(many ? launch_after(s, grid, 256, evict_copy_kernel<4>, a) : launch_after(s, grid, 256, evict_copy_kernel<2>, a));
  LAUNCHED();
  return TSFM_OK;
}

int tsfm_verify_tokens(void *stream, const int32_t *tokens, const float *p, int64_t p_stride, const float *q, int64_t q_stride,
                       int32_t B, int32_t K, int32_t V, const float *u, uint64_t seed, int32_t round_idx, int32_t series0,
                       const int32_t *n_draft, const int32_t *len, int32_t *out, int32_t *n_accept, int32_t *len_out) {
  if (!p || !out || !n_accept || B < 1 || K < 0 || K > TSFM_MAX_K || V < 1 || (K && !tokens) || !len != !len_out) return TSFM_ERR_ARG;
  if (p_stride < V || (q && q_stride < V)) return TSFM_ERR_ARG;
  if (V > kMaxSlots) return TSFM_ERR_SHAPE;
  VerifyArgs a{};
  a.tokens = tokens;
  a.p = p;
  a.q = q;
  a.p_stride = p_stride;
  a.q_stride = q_stride;
  a.K = K;
  a.V = V;
  a.u = u;
  a.key = make_uint2((uint32_t)(seed & 0xffffffffu), (uint32_t)(seed >> 32));
  a.round_idx = round_idx;
  a.series0 = series0;
  a.n_draft = n_draft;
  a.len = len;
  a.out = out;
  a.n_accept = n_accept;
  a.len_out = len_out;
  // All CTAs resident at once where that is possible, 32 warps on an SM in CTAs of four (256 rows of 100003: 4 CTAs of 4 warps each,
  // 7 on an SM; 2 of 8, 3 or 4 on an SM, took a fifth longer); fewer rows get more warps, of 512 entries at least.
  int cluster = 1, warps = 4;
  while (cluster < VERIFY_MAX_CLUSTER && 2ll * B * cluster <= 8 * kSms && V > cluster * 4096) cluster *= 2;
  while (warps < VERIFY_MAX_WARPS && 2ll * B * cluster * warps <= 32 * kSms && V > cluster * warps * 512) warps *= 2;
  if ((long long)B * cluster > kMaxGridX) return TSFM_ERR_SHAPE;
  CU_TRY(launch_cluster((cudaStream_t)stream, (unsigned)(B * cluster), 32 * warps, 0, cluster, verify_tokens_kernel, a));
  LAUNCHED();
  return TSFM_OK;
}

}  // extern "C"
