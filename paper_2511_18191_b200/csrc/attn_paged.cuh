// Attention of a series' new tokens over its cache of pages (tsfm_paged_attention).
//
// Work: a unit is one series, one key head and up to ROWS of its query rows (new tokens x heads of the group: they read the
// same keys).  A unit's slots are cut into tiles, the tiles of all units are numbered through, and every CTA takes an
// equal run of them: lengths may differ by any factor and nothing waits for the longest series.  A unit's tiles are those that any of
// the series' tokens sees, whichever rows it has: with few new tokens that is what its own rows see; with many (a prompt) most of it
// is masked, and units whose rows lie behind n_new read it for nothing.  A run covers at most
// two units in part, its first and its last; those leave (max, sum, unnormalised output) in the workspace, and
// paged_join_kernel joins the parts in order.  Running maximum and sum per row, scores in base 2.
#pragma once
#include "pages.cuh"

namespace tsfm {

constexpr int PA_TILE = 64;                        // slots
constexpr int PA_JOIN_WARPS = 8;

// What a CTA that starts inside a unit leaves for the join: the unit, and the CTAs that share it.
struct PagedMeta {
  int b, u, c0, c1;                                // b < 0: nothing
};

struct PagedAttnArgs {
  PagesDev pg;                                     // capacity: also cut to max_len
  const void *q;
  void *out;
  long long q_stride, out_stride;                  // elements
  const int *len, *n_new;                          // n_new or NULL
  int B, M, n_heads, group;                        // group = n_heads / n_kv_heads
  uint32_t group_magic;                            // ceil(2^32 / group): see token_of
  float scale2;                                    // scale * log2(e)
  int causal, window;
  float *lse;                                      // or NULL
  const float *w_in;                               // or NULL
  float *w_out;                                    // or NULL
  long long w_stride;
  int chunks, units;                               // row chunks of a key head, units of a series
  PagedMeta *meta;                                 // [grid]
  float2 *part_ml;                                 // [2 grid][rows]
  float *part_o;                                   // [2 grid][rows][D]
  float *lse2;                                     // [B][heads of keys][M group], with weights only
  float *scores;                                   // [B][heads of keys][M group][score_stride], with weights only
  long long score_stride;
  unsigned long long wait_ns;                      // limit of a wait for a tile
  int miss_from;                                   // tests: from this tile of a CTA on more bytes are waited for than are copied
  // of trees and windows (attn_tree.cuh) only
  const unsigned long long *mask;                  // [B or 1][M][words], or NULL: a chain
  const int *depth;                                // [B or 1][M], or NULL
  long long mask_series, depth_series;             // from a series to the next: 0 with one tree for all
  int words, sinks;
};

// The token of a query row (row / group).  Rows and groups are below 2^16, so the rounded-up reciprocal is exact.
__device__ __forceinline__ int token_of(const PagedAttnArgs &a, int row) { return a.group == 1 ? row : (int)__umulhi((uint32_t)row, a.group_magic); }

// Unit u of a series: its key head, and which of the head's row chunks it is.
template <bool TREE> __device__ __forceinline__ int paged_unit_head(const PagedAttnArgs &a, int u) { return TREE ? u % a.pg.n_kv_heads : u / a.chunks; }
template <bool TREE> __device__ __forceinline__ int paged_unit_chunk(const PagedAttnArgs &a, int u) { return TREE ? u / a.pg.n_kv_heads : u % a.chunks; }

// A series as this call sees it: its live rows, the slots that any of them sees, the tiles that hold those.
struct PagedSpan {
  int len, n_new, total, lo, tile0, tiles;
};
__device__ __forceinline__ PagedSpan paged_span_of(const PagedAttnArgs &a, int raw, int raw_new, bool report) {
  PagedSpan s;
  s.len = cut(raw, a.pg.capacity);
  s.n_new = cut(raw_new, a.M);
  const long long total = (long long)s.len + (a.causal ? s.n_new : 0);
  s.total = (int)min(total, (long long)a.pg.capacity);
  if (report && (raw != s.len || total != s.total)) pages_report(a.pg, BAD_LEN);
  const int first_end = a.causal ? min(s.len + 1, s.total) : s.total;
  s.lo = a.window ? max(0, first_end - a.window) : 0;
  s.tile0 = s.lo / PA_TILE;
  // a live row without slots still has an answer: one tile
  s.tiles = s.n_new == 0 ? 0 : max(1, (s.total + PA_TILE - 1) / PA_TILE - s.tile0);
  return s;
}
__device__ __forceinline__ PagedSpan paged_span(const PagedAttnArgs &a, int b, bool report) {
  return paged_span_of(a, __ldg(a.len + b), a.n_new ? __ldg(a.n_new + b) : a.M, report);
}
// Slots [lo, end) that row m sees.
__device__ __forceinline__ int2 paged_row_range(const PagedAttnArgs &a, const PagedSpan &s, int m) {
  const int end = m >= s.n_new ? 0 : a.causal ? min(s.len + m + 1, s.total) : s.total;
  return make_int2(a.window ? max(0, end - a.window) : 0, end);
}

// The tile after (b, u, t) in a run, next() the span of the series after b's last one.  Bounded by B and units: should a length change under
// a call, which nobody may let happen, the walk stays at the last series and the call ends.
#pragma nv_exec_check_disable
template <typename F>
__host__ __device__ __forceinline__ void paged_next_tile(int &b, int &u, int &t, PagedSpan &sp, int B, int units, F next) {
  if (++t < sp.tiles) return;
  t = 0;
  if (++u < units) return;
  u = 0;
  while (b + 1 < B) {
    ++b;
    sp = next();
    if (sp.tiles) break;
  }
}

// The CTA's run of tiles: `count` of them from tile `first` of unit `u` of series `b`; per: tiles a CTA; unit0: number of that
// unit's first tile.
struct PagedRun {
  int b, u, first, count;
  long long unit0, per;
};
// Every thread sums the tiles of a contiguous share of the series, a block scan places them.
template <int THREADS>
__device__ PagedRun paged_find_run(const PagedAttnArgs &a) {
  __shared__ long long warp_sum_s[THREADS / 32];
  __shared__ PagedRun found;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int share = (a.B + THREADS - 1) / THREADS, b0 = min(a.B, tid * share), b1 = min(a.B, b0 + share);
  long long mine = 0;
  for (int b = b0; b < b1; ++b) mine += (long long)paged_span(a, b, blockIdx.x == 0).tiles * a.units;
  long long inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += v;
  }
  if (lane == 31) warp_sum_s[warp] = inc;
  if (tid == 0) found.b = -1, found.count = 0;
  __syncthreads();
  long long before = inc - mine, total = 0;
  for (int i = 0; i < THREADS / 32; ++i) {
    if (i < warp) before += warp_sum_s[i];
    total += warp_sum_s[i];
  }
  const long long per = max(1ll, (total + gridDim.x - 1) / gridDim.x), start = per * blockIdx.x;
  if (start >= before && start < before + mine) {
    for (int b = b0; b < b1; ++b) {
      const int tiles = paged_span(a, b, false).tiles;
      const long long here = (long long)tiles * a.units;
      if (start < before + here) {
        const int u = (int)((start - before) / tiles), first = (int)((start - before) - (long long)u * tiles);
        found = PagedRun{b, u, first, (int)min(per, total - start), start - first, per};
        break;
      }
      before += here;
    }
  }
  __syncthreads();
  return found;
}

// Where a row's result goes: straight to the caller, or as a part into the workspace.
__device__ __forceinline__ void paged_write_lse(const PagedAttnArgs &a, int b, int h, int row, float m, float l) {
  const int tok = token_of(a, row), head = h * a.group + row - tok * a.group;
  const float lse2 = l == 0.f ? -INFINITY : m + log2f(l);
  if (a.lse) a.lse[((long long)b * a.M + tok) * a.n_heads + head] = lse2 * 0.69314718055994530942f;
  if (a.lse2) a.lse2[((long long)b * a.pg.n_kv_heads + h) * a.M * a.group + row] = lse2;
}
template <typename T>
__device__ __forceinline__ T *paged_out_row(const PagedAttnArgs &a, int b, int h, int row, int D) {
  const int tok = token_of(a, row), head = h * a.group + row - tok * a.group;
  return reinterpret_cast<T *>(a.out) + ((long long)b * a.M + tok) * a.out_stride + (long long)head * D;
}

// Joins the parts of the units that several CTAs shared: block x belongs to CTA x of the kernel before and works if that one is
// the second of a unit's CTAs; the y blocks share its rows.  Eight warps: each a row where a unit has few parts, all of them one
// row where it has many (one series of 131071 slots has 37: a warp alone made them a chain of loads as long as a third of the
// kernel before).
// TREE: units are numbered as attn_tree.cuh does it.
template <typename T, int D, bool TREE>
__global__ void __launch_bounds__(32 * PA_JOIN_WARPS) paged_join_kernel(const __grid_constant__ PagedAttnArgs a, int ROWS) {
  constexpr int E = D / 32, W = PA_JOIN_WARPS;
  __shared__ float s_o[W][D];
  __shared__ float2 s_ml[W];
  pdl_sync();
  const PagedMeta meta = a.meta[blockIdx.x];
  if (meta.b < 0 || meta.c0 + 1 != (int)blockIdx.x) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int h = paged_unit_head<TREE>(a, meta.u), row0 = paged_unit_chunk<TREE>(a, meta.u) * ROWS;
  const int n_new = a.n_new ? cut(a.n_new[meta.b], a.M) : a.M;
  const int rows = min(min(ROWS, a.M * a.group - row0), n_new * a.group - row0);       // live ones
  const int parts = meta.c1 - meta.c0 + 1;
  const bool alone = parts <= 8;                   // a warp a row
  const int share = alone ? 1 : W, sub = alone ? 0 : warp;
  for (int r0 = blockIdx.y * (W / share); r0 < rows; r0 += gridDim.y * (W / share)) {
    const int r = r0 + (alone ? warp : 0);
    auto index = [&](int i) { return (long long)(i == 0 ? 2 * meta.c0 + 1 : 2 * (meta.c0 + i)) * ROWS + r; };
    float top = -INFINITY, sum = 0.f, o[E] = {};
#pragma unroll 1
    for (int i0 = sub; i0 < parts && r < rows; i0 += 4 * share) {
      float2 ml[4];
      float x[4][E];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = i0 + j * share;
        ml[j] = i < parts ? a.part_ml[index(i)] : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int e = 0; e < E; ++e) x[j][e] = i < parts ? a.part_o[index(i) * D + e * 32 + lane] : 0.f;
      }
      float now = top;
#pragma unroll
      for (int j = 0; j < 4; ++j) now = fmaxf(now, ml[j].x);
      const float ref = now == -INFINITY ? 0.f : now, f0 = exp2f(top - ref);
      top = now;
      sum *= f0;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] *= f0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float f = exp2f(ml[j].x - ref);
        sum = fmaf(ml[j].y, f, sum);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(x[j][e], f, o[e]);
      }
    }
    if (!alone) {
      __syncthreads();
      if (lane == 0) s_ml[warp] = make_float2(top, sum);
#pragma unroll
      for (int e = 0; e < E; ++e) s_o[warp][e * 32 + lane] = o[e];
      __syncthreads();
      if (warp) continue;
      top = s_ml[0].x;
#pragma unroll
      for (int w = 1; w < W; ++w) top = fmaxf(top, s_ml[w].x);
      const float ref = top == -INFINITY ? 0.f : top;
      sum = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = exp2f(s_ml[w].x - ref);
        sum = fmaf(s_ml[w].y, f, sum);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(s_o[w][e * 32 + lane], f, o[e]);
      }
    }
    if (r >= rows) continue;
    T *out = paged_out_row<T>(a, meta.b, h, row0 + r, D);
#pragma unroll
    for (int e = 0; e < E; ++e) out[e * 32 + lane] = from_f32<T>(sum == 0.f ? 0.f : o[e] / sum);
    if (lane == 0) paged_write_lse(a, meta.b, h, row0 + r, top, sum);
  }
}

// w_out = w_in + sum over the rows of 2^(score - lse2); a slot that a row does not see has the score -inf there.  A row whose lse2 is NaN
// (its query, or a key that it sees, is not finite) gives NaN to the slots that it sees, by their place, and nothing to the others.  A thread
// four slots, eight rows of scores in flight.
constexpr int PA_WEIGHT_ROWS = 64;
__global__ void __launch_bounds__(128, 7) paged_weights_kernel(const __grid_constant__ PagedAttnArgs a) {
  __shared__ float s_lse[PA_WEIGHT_ROWS];
  __shared__ unsigned s_nan[2];
  static_assert(PA_WEIGHT_ROWS == 64, "two warps look them over");
  pdl_wait();
  const int Hkv = a.pg.n_kv_heads, b = blockIdx.x / Hkv, R = a.M * a.group;
  const PagedSpan s = paged_span(a, b, false);
  const float *w_in = a.w_in ? a.w_in + blockIdx.x * a.w_stride : nullptr;
  float *w_out = a.w_out + blockIdx.x * a.w_stride;
  const int live = s.n_new * a.group;
  for (int base = blockIdx.y * 512; base < s.total; base += gridDim.y * 512) {
    const int slot = base + threadIdx.x * 4;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < live; r0 += PA_WEIGHT_ROWS) {
      __syncthreads();
      if (threadIdx.x < PA_WEIGHT_ROWS) {          // (a row that got nothing gives nothing)
        const float lse2 = r0 + threadIdx.x < live ? a.lse2[(long long)blockIdx.x * R + r0 + threadIdx.x] : INFINITY;
        const unsigned bad = __ballot_sync(0xffffffffu, isnan(lse2));
        if (threadIdx.x % 32 == 0) s_nan[threadIdx.x / 32] = bad;
        s_lse[threadIdx.x] = lse2 == -INFINITY || isnan(lse2) ? INFINITY : lse2;
      }
      __syncthreads();
      unsigned long long nan = s_nan[0] | (unsigned long long)s_nan[1] << 32;
      if (slot >= s.total || slot < s.tile0 * PA_TILE) continue;       // before the first tile nothing was seen
      const float *src = a.scores + ((long long)blockIdx.x * R + r0) * a.score_stride + slot;
      const int n = min(PA_WEIGHT_ROWS, live - r0);
      for (int r = 0; r < n; r += 8) {
        float4 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = r + j < n ? *reinterpret_cast<const float4 *>(src + (r + j) * a.score_stride) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float lse2 = r + j < n ? s_lse[r + j] : INFINITY;
          w[0] += exp2f(v[j].x - lse2), w[1] += exp2f(v[j].y - lse2), w[2] += exp2f(v[j].z - lse2), w[3] += exp2f(v[j].w - lse2);
        }
      }
      for (; nan; nan &= nan - 1) {                // (seldom)
        const int2 sees = paged_row_range(a, s, token_of(a, r0 + __ffsll(nan) - 1));
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (slot + e >= sees.x && slot + e < sees.y && page_of(a.pg, a.pg.table + (long long)b * a.pg.table_stride, slot + e) >= 0) w[e] = NAN;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (slot + e < s.total) w_out[slot + e] = (w_in ? w_in[slot + e] : 0.f) + w[e];
  }
}

}  // namespace tsfm
