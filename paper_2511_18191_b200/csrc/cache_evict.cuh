// Eviction by accumulated attention weight (tsfm_cache_evict): which slots a head keeps, then the copy of their keys and
// values into other pages.
#pragma once
#include <cooperative_groups.h>
#include "pages.cuh"

namespace tsfm {

struct EvictArgs {
  PagesDev pg;
  const int *dst_table;
  int dst_stride;
  const int *len;
  const float *w;
  long long w_stride, w_out_stride;
  int B, budget, sinks, recent;
  int *kept;                                       // [B, heads, budget]
  float *w_out;                                    // or NULL
  int *len_out;
  int vecs;                                        // 16-byte vectors of a row
};

// Weights as unsigned numbers in the same order; -0 equals 0, NaN lies below -inf.
__device__ __forceinline__ uint32_t weight_rank(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  if (isnan(w)) return 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One CTA, or a cluster of them where it is long, a series and head.  Sinks and recent slots get a rank above all others; then the
// budget-th largest rank by three rounds of counting, digits of 11, 11 and 10 bits from the top; then the kept slots' places.  A warp
// owns a contiguous part of the slots, whose ranks stay in shared memory where they fit (16 slots a thread).  Loops stay loops: with
// the ranks in registers, hence every pass unrolled, fetching the code took longer than running it.  The counters have copies, by
// lane: the top digits of a heavy-tailed distribution are few.
// Bound: the chain of rounds for one series (4 heads of 4100 slots: 8 us), instructions for many (32 x 8 heads of up to 16384 slots:
// 32 us).
constexpr int EVICT_MAX_CLUSTER = 8, EVICT_BINS = 2048;

template <int THREADS> struct EvictShared {
  static constexpr int WARPS = THREADS / 32, OWN = 16 * THREADS, COPIES = THREADS / 256;       // OWN: slots that a CTA holds
  int bins[COPIES][EVICT_BINS], warp_hi[WARPS], warp_eq[WARPS];
  int all_hi[EVICT_MAX_CLUSTER], all_eq[EVICT_MAX_CLUSTER];
  uint32_t found;
  int left;
  uint2 mask[OWN / 32];                            // of 32 slots: those above the threshold, those equal to it
  uint32_t rank[OWN];
};

// KEPT: all of the series' ranks are in shared memory.
template <bool KEPT, int THREADS>
__device__ __forceinline__ void evict_select(const EvictArgs &a, EvictShared<THREADS> &sh, const float *w, int n, int *kept) {
  constexpr int WARPS = EvictShared<THREADS>::WARPS, OWN = EvictShared<THREADS>::OWN, COPIES = EvictShared<THREADS>::COPIES;
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, C = (int)cluster.num_blocks(), c = (int)cluster.block_rank();
  const int lo = a.sinks, hi = n - a.recent;
  const long long part = ((n + C * WARPS - 1) / (C * WARPS) + 31) / 32 * 32;
  const int p0 = (int)min((long long)n, (c * WARPS + warp) * part), p1 = (int)min((long long)n, p0 + part);
  uint32_t *const own = sh.rank + warp * (OWN / WARPS) + lane;       // of slots p0 + lane, p0 + lane + 32, ..
  uint2 *const masks = sh.mask + warp * (OWN / 32 / WARPS);
  auto rank_of = [&](int i) { return i < lo || i >= hi ? 0xffffffffu : weight_rank(w[i]); };
  if (KEPT) {
#pragma unroll 8
    for (int i = p0 + lane; i < p1; i += 32) own[i - lane - p0] = rank_of(i);
    __syncwarp();
  }
  // f(number of the group, rank, whether the slot is one) for the warp's slots, 32 at a time
  auto each = [&](auto f) {
#pragma unroll 4
    for (int i = p0; i < p1; i += 32) {
      const bool in = i + lane < p1;
      f((i - p0) >> 5, !in ? 0u : KEPT ? own[i - p0] : rank_of(i + lane), in);
    }
  };
  uint32_t prefix = 0;                             // bits of the threshold so far
  int eq_need = a.budget;                          // of the slots with that prefix, how many are kept
  int shift = 32;
#pragma unroll 1
  for (int round = 0; round < 3; ++round) {
    const int bits = round == 2 ? 10 : 11;
    const uint32_t above = round ? 0xffffffffu << shift : 0, digit = (1u << bits) - 1;       // bits that are known; the next ones
    shift -= bits;
    for (int i = tid; i < COPIES * EVICT_BINS / 4; i += THREADS) reinterpret_cast<int4 *>(sh.bins)[i] = make_int4(0, 0, 0, 0);
    __syncthreads();
    int *const bins = sh.bins[lane % COPIES];
    each([&](int, uint32_t r, bool in) {
      if (in && (r & above) == prefix) atomicAdd(bins + (r >> shift & digit), 1);
    });
    __syncthreads();
    // thread t owns the PER bins that are t-th from the top
    constexpr int PER = EVICT_BINS / THREADS;
    const int top = EVICT_BINS - 1 - PER * tid;
    int mine[PER], sum = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      mine[j] = 0;
#pragma unroll
      for (int k = 0; k < COPIES; ++k) mine[j] += sh.bins[k][top - j];
    }
    if (C > 1) {
#pragma unroll
      for (int j = 0; j < PER; ++j) sh.bins[0][top - j] = mine[j];
      cluster.sync();
#pragma unroll
      for (int j = 0; j < PER; ++j) mine[j] = 0;
      for (int k = 0; k < C; ++k) {
        const int *theirs = cluster.map_shared_rank(sh.bins[0], k);
#pragma unroll
        for (int j = 0; j < PER; ++j) mine[j] += theirs[top - j];
      }
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) sum += mine[j];
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    if (lane == 31) sh.warp_hi[warp] = inc;
    __syncthreads();
    int before = __reduce_add_sync(0xffffffffu, lane < warp ? sh.warp_hi[lane] : 0) + inc - sum;
    if (before < eq_need && eq_need <= before + sum) {
      int j = 0;
#pragma unroll
      for (int k = 0; k < PER - 1; ++k)
        if (j == k && before + mine[k] < eq_need) before += mine[k], ++j;
      sh.found = prefix | (uint32_t)(top - j) << shift;
      sh.left = eq_need - before;
    }
    if (C > 1) cluster.sync();                     // (the others have read this CTA's counts)
    else __syncthreads();
    prefix = sh.found;
    eq_need = sh.left;
  }

  // places: the counts of each warp's part, then of all before it; the warps of all CTAs are in slot order
  int hi_n = 0, eq_n = 0;
  each([&](int g, uint32_t r, bool in) {
    const unsigned hi_m = __ballot_sync(0xffffffffu, in && r > prefix), eq_m = __ballot_sync(0xffffffffu, in && r == prefix);
    if (KEPT && lane == 0) masks[g] = make_uint2(hi_m, eq_m);
    hi_n += __popc(hi_m);
    eq_n += __popc(eq_m);
  });
  if (lane == 0) sh.warp_hi[warp] = hi_n, sh.warp_eq[warp] = eq_n;
  __syncthreads();
  int hi_at = __reduce_add_sync(0xffffffffu, lane < warp ? sh.warp_hi[lane] : 0);
  int eq_at = __reduce_add_sync(0xffffffffu, lane < warp ? sh.warp_eq[lane] : 0);
  if (C > 1) {
    if (warp == WARPS - 1 && lane < C) {
      *cluster.map_shared_rank(&sh.all_hi[c], lane) = hi_at + hi_n;
      *cluster.map_shared_rank(&sh.all_eq[c], lane) = eq_at + eq_n;
    }
    cluster.sync();
    hi_at += __reduce_add_sync(0xffffffffu, lane < c ? sh.all_hi[lane] : 0);
    eq_at += __reduce_add_sync(0xffffffffu, lane < c ? sh.all_eq[lane] : 0);
  }
  const unsigned bit = 1u << lane, below = bit - 1;
  auto place = [&](int i, unsigned hi_m, unsigned eq_m) {
    const int eq_here = eq_at + __popc(eq_m & below);            // equal slots before this one: the lowest eq_need stay
    if ((hi_m & bit) || ((eq_m & bit) && eq_here < eq_need)) kept[hi_at + __popc(hi_m & below) + min(eq_here, eq_need)] = i;
    hi_at += __popc(hi_m);
    eq_at += __popc(eq_m);
  };
  if (KEPT) {
#pragma unroll 4
    for (int i = p0; i < p1; i += 32) {
      const uint2 m = masks[(i - p0) >> 5];
      place(i + lane, m.x, m.y);
    }
  } else {
    each([&](int g, uint32_t r, bool in) {
      const unsigned hi_m = __ballot_sync(0xffffffffu, in && r > prefix), eq_m = __ballot_sync(0xffffffffu, in && r == prefix);
      place(p0 + 32 * g + lane, hi_m, eq_m);
    });
  }
}

// (a cluster only where the longest series' ranks take more than one CTA's shared memory)
template <int THREADS>
__global__ void __launch_bounds__(THREADS, 2048 / THREADS) evict_select_kernel(EvictArgs a) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  extern __shared__ __align__(16) unsigned char evict_smem[];
  EvictShared<THREADS> &sh = *reinterpret_cast<EvictShared<THREADS> *>(evict_smem);
  const int C = (int)cluster.num_blocks(), c = (int)cluster.block_rank(), pair = blockIdx.x / C;
  const int Hkv = a.pg.n_kv_heads, b = pair / Hkv, tid = threadIdx.x;
  const int raw = a.len[b], n = cut(raw, a.pg.capacity);
  const int keep = min(n, a.budget);
  if (pair % Hkv == 0 && tid == 0 && c == 0) {
    a.len_out[b] = keep;
    if (raw != n) pages_report(a.pg, BAD_LEN);
  }
  const float *w = a.w + pair * a.w_stride;
  int *kept = a.kept + (long long)pair * a.budget;
  for (int j = keep + c * THREADS + tid; j < a.budget; j += C * THREADS) kept[j] = -1;
  if (n <= a.budget) {
    for (int j = c * THREADS + tid; j < n; j += C * THREADS) kept[j] = j;
  } else {
    if (C > 1) cluster.sync();                     // (all of them run before one reads another's shared memory)
    if (n <= C * sh.OWN) evict_select<true>(a, sh, w, n, kept);
    else evict_select<false>(a, sh, w, n, kept);
    if (C > 1) cluster.sync();                     // (nor leaves before)
  }
}

// Rows of keys and values of the kept slots, 16 bytes a thread, EVICT_ROWS rows each, and their weights.  Bound: memory, where there are
// many (32 x 8 heads of up to 2048 rows of 256 bytes, 512 MB read and written: 83.5 us, 6.1 TB/s; rows one after the other, 103).
template <int EVICT_ROWS>
__global__ void __launch_bounds__(256, EVICT_ROWS == 4 ? 4 : 6) evict_copy_kernel(EvictArgs a) {
  pdl_wait();
  const int Hkv = a.pg.n_kv_heads, h = blockIdx.x % Hkv, b = blockIdx.x / Hkv;
  const int vec = threadIdx.x & (a.vecs - 1), row = threadIdx.x / a.vecs, rows = 256 / a.vecs;
  const int keep = min(cut(a.len[b], a.pg.capacity), a.budget);
  const int *kept = a.kept + (long long)blockIdx.x * a.budget;
  const float *w = a.w + blockIdx.x * a.w_stride;
  float *w_out = a.w_out ? a.w_out + blockIdx.x * a.w_out_stride : nullptr;
  const int *src_row = a.pg.table + (long long)b * a.pg.table_stride, *dst_row = a.dst_table + (long long)b * a.dst_stride;
  int bad = 0;
  for (int j0 = blockIdx.y * rows * EVICT_ROWS + row; j0 < keep; j0 += gridDim.y * rows * EVICT_ROWS) {
    // each step of the chain place - slot - pages - rows for all of them at once
    int slot[EVICT_ROWS], from[EVICT_ROWS], dst[EVICT_ROWS];
    uint4 k[EVICT_ROWS], v[EVICT_ROWS];
    float weight[EVICT_ROWS];
#pragma unroll
    for (int r = 0; r < EVICT_ROWS; ++r) slot[r] = j0 + r * rows < keep ? kept[j0 + r * rows] : -1;
#pragma unroll
    for (int r = 0; r < EVICT_ROWS; ++r) {
      from[r] = slot[r] < 0 ? 0 : page_of(a.pg, src_row, slot[r]);
      dst[r] = slot[r] < 0 ? 0 : page_of(a.pg, dst_row, j0 + r * rows);
      weight[r] = slot[r] >= 0 && vec == 0 && w_out ? w[slot[r]] : 0.f;
    }
#pragma unroll
    for (int r = 0; r < EVICT_ROWS; ++r) {
      if (from[r] < 0 || dst[r] < 0) bad = BAD_ID;
      else if (slot[r] >= 0) {
        const long long at = slot_offset(a.pg, from[r], h, slot[r]) + vec * 16;
        k[r] = *reinterpret_cast<const uint4 *>(a.pg.k + at);
        v[r] = *reinterpret_cast<const uint4 *>(a.pg.v + at);
      }
    }
#pragma unroll
    for (int r = 0; r < EVICT_ROWS; ++r) {
      if (slot[r] < 0) continue;
      if (vec == 0 && w_out) w_out[j0 + r * rows] = weight[r];
      if (from[r] < 0 || dst[r] < 0) continue;
      const long long to = slot_offset(a.pg, dst[r], h, j0 + r * rows) + vec * 16;
      *reinterpret_cast<uint4 *>(a.pg.k + to) = k[r];
      *reinterpret_cast<uint4 *>(a.pg.v + to) = v[r];
    }
  }
  if (bad) pages_report(a.pg, bad);
}

}  // namespace tsfm
