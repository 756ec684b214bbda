// Eviction by accumulated attention weight (tsfm_cache_evict): which slots a head keeps, then the copy of their keys and
// values into other pages.
#pragma once
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

// One CTA a series and head.  The `need`-th largest weight of the middle by three rounds of counting, 11, 11 and 10 bits
// of the rank from the top; then one pass that numbers the kept slots in order.  A warp owns a contiguous part of the slots,
// whose weights stay in registers where they fit (16384 slots): read once, all loads in flight, they take a third of the time
// of five passes over L2 (32 x 8 heads of up to 16384 slots: 41 us).
constexpr int EVICT_THREADS = 1024, EVICT_BINS = 2048, EVICT_KEEP = 16;
template <bool KEPT> struct EvictWeights {
  const float *w;
  int p0, p1, lane;
  float own[KEPT ? EVICT_KEEP : 1];
  __device__ __forceinline__ void load() {
    if (KEPT)
#pragma unroll
      for (int j = 0; j < EVICT_KEEP; ++j) own[j] = p0 + 32 * j + lane < p1 ? w[p0 + 32 * j + lane] : 0.f;
  }
  // f(slot, weight, whether the slot is one) for this lane's slots, 32 of the warp's at a time in ascending order
  template <typename F> __device__ __forceinline__ void each(F f) const {
    if (KEPT) {
#pragma unroll
      for (int j = 0; j < EVICT_KEEP; ++j)
        if (p0 + 32 * j < p1) f(p0 + 32 * j + lane, own[j], p0 + 32 * j + lane < p1);
    } else {
      for (int i = p0; i < p1; i += 32 * 8) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = i + 32 * j + lane < p1 ? w[i + 32 * j + lane] : 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (i + 32 * j < p1) f(i + 32 * j + lane, x[j], i + 32 * j + lane < p1);
      }
    }
  }
};

struct EvictShared {
  int bins[EVICT_BINS], warp_hi[32], warp_eq[32];
  uint32_t found;
  int left;
};

template <bool KEPT>
__device__ __forceinline__ void evict_select(const EvictArgs &a, EvictShared &sh, const float *w, int n, int *kept, float *w_out) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int lo = a.sinks, hi = n - a.recent;       // the middle: more than `need` slots
  const int need = a.budget - a.sinks - a.recent;
  const int part = ((n + 31) / 32 + 31) / 32 * 32, p0 = min(n, warp * part);
  EvictWeights<KEPT> ws{w, p0, min(n, p0 + part), lane};
  ws.load();
  uint32_t prefix = 0;                             // bits of the threshold so far
  int eq_need = need;                              // of the slots with that prefix, how many are kept
  if (need > 0) {
    int shift = 32;
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
      const int bits = round == 2 ? 10 : 11;
      const uint32_t above = round ? 0xffffffffu << shift : 0;       // bits that are known
      shift -= bits;
      for (int i = tid; i < EVICT_BINS; i += EVICT_THREADS) sh.bins[i] = 0;
      __syncthreads();
      ws.each([&](int i, float x, bool in) {
        const uint32_t r = weight_rank(x);
        if (in && i >= lo && i < hi && (r & above) == prefix) atomicAdd(&sh.bins[(r >> shift) & ((1u << bits) - 1)], 1);
      });
      __syncthreads();
      // thread t owns the 2 bins that are t-th from the top
      const int top = EVICT_BINS - 1 - 2 * tid;
      const int c1 = sh.bins[top], c0 = sh.bins[top - 1], c = c1 + c0;
      int inc = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += v;
      }
      if (lane == 31) sh.warp_hi[warp] = inc;
      __syncthreads();
      int before = lane < warp ? sh.warp_hi[lane] : 0;
      before = __reduce_add_sync(0xffffffffu, before) + inc - c;
      if (before < eq_need && eq_need <= before + c) {
        const bool second = eq_need > before + c1;
        sh.found = prefix | (uint32_t)(second ? top - 1 : top) << shift;
        sh.left = eq_need - before - (second ? c1 : 0);
      }
      __syncthreads();
      prefix = sh.found;
      eq_need = sh.left;
    }
  }
  // number the kept slots: first the counts of each warp's part, then the places
  auto kind = [&](int i, float x, bool in) {       // 2 kept, 1 equal to the threshold, 0 gone
    if (!in) return 0;
    if (i < lo || i >= hi) return 2;
    if (need == 0) return 0;
    const uint32_t r = weight_rank(x);
    return r > prefix ? 2 : r == prefix ? 1 : 0;
  };
  int hi_n = 0, eq_n = 0;
  ws.each([&](int i, float x, bool in) {
    const int k = kind(i, x, in);
    hi_n += __popc(__ballot_sync(0xffffffffu, k == 2));
    eq_n += __popc(__ballot_sync(0xffffffffu, k == 1));
  });
  __syncthreads();
  if (lane == 0) sh.warp_hi[warp] = hi_n, sh.warp_eq[warp] = eq_n;
  __syncthreads();
  int hi_at = __reduce_add_sync(0xffffffffu, lane < warp ? sh.warp_hi[lane] : 0);
  int eq_at = __reduce_add_sync(0xffffffffu, lane < warp ? sh.warp_eq[lane] : 0);
  const unsigned below = (1u << lane) - 1;
  ws.each([&](int i, float x, bool in) {
    const int k = kind(i, x, in);
    const unsigned hi_m = __ballot_sync(0xffffffffu, k == 2), eq_m = __ballot_sync(0xffffffffu, k == 1);
    const int eq_here = eq_at + __popc(eq_m & below);            // equal slots before this one: the lowest eq_need stay
    if (k == 2 || (k == 1 && eq_here < eq_need)) {
      const int j = hi_at + __popc(hi_m & below) + min(eq_here, eq_need);
      kept[j] = i;
      if (w_out) w_out[j] = x;
    }
    hi_at += __popc(hi_m);
    eq_at += __popc(eq_m);
  });
}

__global__ void __launch_bounds__(EVICT_THREADS) evict_select_kernel(EvictArgs a) {
  __shared__ EvictShared sh;
  const int Hkv = a.pg.n_kv_heads, b = blockIdx.x / Hkv, tid = threadIdx.x;
  const int raw = a.len[b], n = cut(raw, a.pg.capacity);
  const int keep = min(n, a.budget);
  if (blockIdx.x % Hkv == 0 && tid == 0) {
    a.len_out[b] = keep;
    if (raw != n) pages_report(a.pg, BAD_LEN);
  }
  const float *w = a.w + blockIdx.x * a.w_stride;
  int *kept = a.kept + (long long)blockIdx.x * a.budget;
  float *w_out = a.w_out ? a.w_out + blockIdx.x * a.w_out_stride : nullptr;
  for (int j = keep + tid; j < a.budget; j += EVICT_THREADS) kept[j] = -1;
  if (n <= a.budget) {
    for (int j = tid; j < n; j += EVICT_THREADS) {
      kept[j] = j;
      if (w_out) w_out[j] = w[j];
    }
  } else if (n <= EVICT_THREADS * EVICT_KEEP) {
    evict_select<true>(a, sh, w, n, kept, w_out);
  } else {
    evict_select<false>(a, sh, w, n, kept, w_out);
  }
}

// Rows of keys and values of the kept slots, 16 bytes a thread, EVICT_ROWS rows each.
constexpr int EVICT_ROWS = 4;
__global__ void __launch_bounds__(256) evict_copy_kernel(EvictArgs a) {
  pdl_wait();
  const int Hkv = a.pg.n_kv_heads, h = blockIdx.x % Hkv, b = blockIdx.x / Hkv;
  const int vec = threadIdx.x & (a.vecs - 1), row = threadIdx.x / a.vecs, rows = 256 / a.vecs;
  const int keep = min(cut(a.len[b], a.pg.capacity), a.budget);
  const int *kept = a.kept + (long long)blockIdx.x * a.budget;
  const int *src_row = a.pg.table + (long long)b * a.pg.table_stride, *dst_row = a.dst_table + (long long)b * a.dst_stride;
  int bad = 0;
  for (int j0 = blockIdx.y * rows * EVICT_ROWS + row; j0 < keep; j0 += gridDim.y * rows * EVICT_ROWS) {
    uint4 k[EVICT_ROWS], v[EVICT_ROWS];
    long long to[EVICT_ROWS];
#pragma unroll
    for (int r = 0; r < EVICT_ROWS; ++r) {
      const int j = j0 + r * rows;
      to[r] = -1;
      if (j >= keep) continue;
      const int slot = kept[j];
      const int from = page_of(a.pg, src_row, slot), dst = page_of(a.pg, dst_row, j);
      if (from < 0 || dst < 0) {
        bad = BAD_ID;
        continue;
      }
      const long long at = slot_offset(a.pg, from, h, slot) + vec * 16;
      to[r] = slot_offset(a.pg, dst, h, j) + vec * 16;
      k[r] = *reinterpret_cast<const uint4 *>(a.pg.k + at);
      v[r] = *reinterpret_cast<const uint4 *>(a.pg.v + at);
    }
#pragma unroll
    for (int r = 0; r < EVICT_ROWS; ++r) {
      if (to[r] < 0) continue;
      *reinterpret_cast<uint4 *>(a.pg.k + to[r]) = k[r];
      *reinterpret_cast<uint4 *>(a.pg.v + to[r]) = v[r];
    }
  }
  if (bad) pages_report(a.pg, bad);
}

}  // namespace tsfm
