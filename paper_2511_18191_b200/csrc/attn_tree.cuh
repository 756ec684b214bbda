// What a token sees of its series' cache where the new tokens form a tree, or where a sliding window keeps some first slots visible
// (tsfm_tree_attention, tsfm_window_attention), for the kernels of attn_paged_mma.cuh, attn_paged_f32.cuh and attn_tree_tc.cuh.
//
// Token m of a tree stands at position len + depth[m].  Of the slots below len it sees those above its position - window and
// the first `sinks`; of the new tokens' slots len + j those whose bit j is set in its mask.  A chain (mask NULL) is the tree in which
// each token hangs on the one before it, seen as far as the window reaches.
//
// Unlike in attn_paged.cuh every unit (series, row chunk, key head; numbered in this order) has a span of its own: the blocks of 64 slots
// that hold sinks, then those from its first row's window on.  A prompt with a window so reads what its rows see, and chunks behind
// n_new have no tiles.  (256 series, one token of 4 x 8 heads of 128, window 1024 and 4 sinks: 123 us, 5.0 TB/s; 18 tiles a unit, of which each starts with one for the
// sinks alone.)
#pragma once
#include "attn_paged.cuh"

namespace tsfm {

// Blocks of 64 slots before the window's that hold sinks.
__device__ __forceinline__ int paged_sink_tiles(const PagedAttnArgs &a, const PagedSpan &s) { return min((min(a.sinks, s.total) + PA_TILE - 1) / PA_TILE, s.tile0); }
// First slot of a unit's t-th block.
template <bool TREE> __device__ __forceinline__ int paged_tile_base(const PagedAttnArgs &a, const PagedSpan &s, int t) {
  if (!TREE) return (s.tile0 + t) * PA_TILE;
  const int first = paged_sink_tiles(a, s);
  return (t < first ? t : s.tile0 + t - first) * PA_TILE;
}
// Some row of the unit may see one of the n slots from `slot` on.
template <bool TREE> __device__ __forceinline__ bool paged_wants(const PagedAttnArgs &a, const PagedSpan &s, int slot, int n) {
  return slot < s.total && (slot + n > s.lo || (TREE && slot < a.sinks));
}

// Blocks of a unit.
__device__ __forceinline__ int paged_unit_blocks(const PagedAttnArgs &a, const PagedSpan &s) {
  return max(1, paged_sink_tiles(a, s) + max(0, (s.total + PA_TILE - 1) / PA_TILE - s.tile0));
}
// Span of a row chunk of a series.  lo, total: bounds of what its rows see, sinks aside.  PAIR: blocks of a tile.
template <int PAIR = 1>
__device__ __forceinline__ PagedSpan paged_unit_span(const PagedAttnArgs &a, int raw, int raw_new, int chunk, int rows, bool report) {
  PagedSpan s;
  s.len = cut(raw, a.pg.capacity);
  s.n_new = cut(raw_new, a.M);
  const long long all = (long long)s.len + s.n_new;
  s.total = (int)min(all, (long long)a.pg.capacity);
  if (report && (raw != s.len || all != s.total)) pages_report(a.pg, BAD_LEN);
  const int m0 = token_of(a, chunk * rows), m1 = min(s.n_new, token_of(a, min(a.M * a.group, (chunk + 1) * rows) - 1) + 1);
  if (!a.mask) s.total = min(s.total, s.len + m1);
  s.lo = a.window ? max(0, a.mask ? min(s.len, s.len + 1 - a.window) : s.len + m0 + 1 - a.window) : 0;
  s.tile0 = s.lo / PA_TILE;
  // (a live row without slots still has an answer: one tile)
  s.tiles = m0 >= s.n_new ? 0 : (paged_unit_blocks(a, s) + PAIR - 1) / PAIR;
  return s;
}
template <int PAIR = 1> __device__ __forceinline__ PagedSpan paged_unit_span(const PagedAttnArgs &a, int b, int chunk, int rows, bool report) {
  return paged_unit_span<PAIR>(a, __ldg(a.len + b), a.n_new ? __ldg(a.n_new + b) : a.M, chunk, rows, report);
}

// The tile after (b, u, t) in a run; len, n_new: of series b, next() fetches those of the series behind.  Bounded by the series as
// paged_next_tile is.
template <int PAIR = 1, typename F>
__device__ __forceinline__ void paged_next_unit_tile(const PagedAttnArgs &a, int rows, int &b, int &u, int &t, PagedSpan &sp, const int &len, const int &n_new, F next) {
  if (++t < sp.tiles) return;
  t = 0;
  if (++u < a.units) {
    if (u % a.pg.n_kv_heads) return;               // another head's rows of the same chunk
    sp = paged_unit_span<PAIR>(a, len, n_new, u / a.pg.n_kv_heads, rows, false);
    if (sp.tiles) return;                          // (chunks behind one without live rows have none either)
  }
  u = 0;
  while (b + 1 < a.B) {
    ++b;
    next();
    sp = paged_unit_span<PAIR>(a, len, n_new, 0, rows, false);
    if (sp.tiles) break;
  }
}

// As paged_find_run, over the chunks of all series: every thread sums up a contiguous share of them.  What starts and ends a unit counts as
// `start` tiles, in front of its own, so that runs of many short units are as long as those of few long ones.  (unit0: place of the unit's first
// tile on this scale.)
template <int THREADS, int PAIR = 1>
__device__ PagedRun paged_find_unit_run(const PagedAttnArgs &a, int rows, int start) {
  __shared__ long long warp_sum_s[2][THREADS / 32];
  __shared__ PagedRun found;
  __shared__ long long tiles_to[2];                // tiles before the run, before its end
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, Hkv = a.pg.n_kv_heads;
  const long long items = (long long)a.B * a.chunks, share = (items + THREADS - 1) / THREADS;
  const long long i0 = min(items, tid * share), i1 = min(items, i0 + share);
  auto each = [&](auto f) {                        // f(series, chunk, tiles of one head)
    int b = (int)(i0 / a.chunks), c = (int)(i0 - (long long)b * a.chunks);
    int len = 0, n_new = 0;
    for (long long i = i0; i < i1; ++i) {
      if (i == i0 || c == 0) len = __ldg(a.len + b), n_new = a.n_new ? __ldg(a.n_new + b) : a.M;
      f(b, c, paged_unit_span<PAIR>(a, len, n_new, c, rows, false).tiles);
      if (++c == a.chunks) c = 0, ++b;
    }
  };
  long long mine = 0, own_tiles = 0;
  each([&](int b, int c, int tiles) {
    own_tiles += (long long)tiles * Hkv;
    mine += tiles ? (long long)(tiles + start) * Hkv : 0;
  });
  if (blockIdx.x == 0)
    for (int b = tid; b < a.B; b += THREADS) paged_unit_span<PAIR>(a, b, 0, rows, true);
  long long inc = mine, tiles_inc = own_tiles;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, inc, o), w = __shfl_up_sync(0xffffffffu, tiles_inc, o);
    if (lane >= o) inc += v, tiles_inc += w;
  }
  if (lane == 31) warp_sum_s[0][warp] = inc, warp_sum_s[1][warp] = tiles_inc;
  if (tid == 0) found.b = -1;
  __syncthreads();
  long long before = inc - mine, tiles_before = tiles_inc - own_tiles, total = 0, all_tiles = 0;
  for (int i = 0; i < THREADS / 32; ++i) {
    if (i < warp) before += warp_sum_s[0][i], tiles_before += warp_sum_s[1][i];
    total += warp_sum_s[0][i];
    all_tiles += warp_sum_s[1][i];
  }
  const long long per = max(1ll, (total + gridDim.x - 1) / gridDim.x), begin = per * blockIdx.x, end = begin + per;
  if (tid == 0) {
    if (begin >= total) tiles_to[0] = all_tiles;
    if (end >= total) tiles_to[1] = all_tiles;
  }
  if ((begin >= before && begin < before + mine) || (end >= before && end < before + mine)) {
    each([&](int b, int c, int tiles) {
      const long long unit = tiles ? tiles + start : 0, here = unit * Hkv;
      for (int x = 0; x < 2; ++x) {
        const long long at = x ? end : begin;
        if (at < before || at >= before + here) continue;
        const int h = (int)((at - before) / unit), first = (int)((at - before) - h * unit);
        tiles_to[x] = tiles_before + (long long)h * tiles + max(0, first - start);
        if (!x) found = PagedRun{b, c * Hkv + h, max(0, first - start), 0, before + h * unit + start, per};
      }
      before += here;
      tiles_before += (long long)tiles * Hkv;
    });
  }
  __syncthreads();
  PagedRun run = found;
  run.count = (int)(tiles_to[1] - tiles_to[0]);
  return run;
}

// Slots [x, y) are the window of token m, in a tree below len.
__device__ __forceinline__ int2 paged_tree_range(const PagedAttnArgs &a, const PagedSpan &s, int b, int m) {
  if (m >= s.n_new) return make_int2(0, 0);
  if (!a.mask) return make_int2(a.window ? max(0, s.len + m + 1 - a.window) : 0, min(s.len + m + 1, s.total));
  return make_int2(a.window ? max(0, s.len + cut(__ldg(a.depth + b * a.depth_series + m), a.M - 1) + 1 - a.window) : 0, s.len);
}
// Slots [x, y) that every one of the tokens m0 .. last sees.
__device__ __forceinline__ int2 paged_tree_open(const PagedAttnArgs &a, const PagedSpan &s, int m0, int last) {
  return make_int2(a.window ? max(0, s.len + (a.mask ? a.M - 1 : last) + 1 - a.window) : 0, a.mask ? s.len : min(s.len + m0 + 1, s.total));
}

// Bits lo .. hi - 1, as far as they are among 64.
__device__ __forceinline__ unsigned long long bits_between(int lo, int hi) {
  lo = max(lo, 0);
  hi = min(hi, 64);
  return lo < hi ? ~0ull >> (64 - (hi - lo)) << lo : 0ull;
}
// Which of the slots base .. base + 63 token m sees (m >= n_new: none), range as paged_tree_range gives it.
__device__ __forceinline__ unsigned long long paged_tree_bits(const PagedAttnArgs &a, const PagedSpan &s, int2 range, int b, int m, int base) {
  if (m >= s.n_new) return 0ull;
  unsigned long long bits = bits_between(range.x - base, range.y - base) | bits_between(-base, min(a.sinks, range.y) - base);
  if (a.mask && base + 64 > s.len) {
    const unsigned long long *row = a.mask + b * a.mask_series + (long long)m * a.words;
    const int at = base - s.len, w = at >> 6, shift = at & 63;         // (rounds down: w is -1 where the tile begins before len)
    const unsigned long long x0 = w >= 0 && w < a.words ? __ldg(row + w) : 0ull, x1 = shift && w + 1 < a.words ? __ldg(row + w + 1) : 0ull;
    bits |= (x0 >> shift | (shift ? x1 << (64 - shift) : 0ull)) & bits_between(s.len - base, s.total - base);
  }
  return bits;
}

}  // namespace tsfm
