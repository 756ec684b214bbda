// A token drawn from a row of weights by inverse CDF, by a cluster of CTAs (tsfm_verify_tokens, tsfm_verify_tree).
//
// CTA c, and in it each warp, sums a contiguous part of the row, and keeps the sums of up to 32 segments of it.  The draw then falls
// into a CTA's, a warp's, a segment's part: 256 entries for rows of up to 32 x 256 a warp, which one warp looks through; a longer segment is
// shared by the CTA's warps as the row was.  Sums are fp64 so that their order decides nothing.
#pragma once
#include <cooperative_groups.h>
#include "accept.cuh"

namespace tsfm {

constexpr int VERIFY_MAX_WARPS = 16, VERIFY_MAX_CLUSTER = 8, VERIFY_BATCH = 256;

// A probability as a weight of the draw: what is negative or not finite counts as 0.  (The bits of a positive finite float are
// 1 .. 0x7f7fffff.)
__device__ __forceinline__ float draw_weight(float p) { return __float_as_uint(p) - 1u < 0x7f7fffffu ? p : 0.f; }
// A uniform as both calls read it.
__device__ __forceinline__ double draw_uniform(float u) { return (double)fminf(fmaxf(u, 0.f), 0.999999940395355224609375f); }

// Sums of ROW over [lo, hi) by a warp, one of every `length` entries (a multiple of 256) into seg[], and all of them, in all lanes.
// row.fetch<Q>: entries t, t + 32, .. of a lane, those at or behind `hi` as nothing; row.weight: what they count.  Q: the row has a second part.
// Sixteen loads of a lane in flight (eight without q): with what the compiler had gathered by itself the batch of 256 rows of 100003 took 132 us.
template <bool Q, typename Row>
__device__ __forceinline__ double row_sums(const Row &row, int lo, int hi, int length, int lane, double *seg) {
  constexpr int N = VERIFY_BATCH / 32;
  double total = 0;
  const float *pt = row.p + lo + lane, *qt = Q ? row.q + lo + lane : nullptr;
  for (int k = 0; lo < hi; ++k) {
    double s[4] = {0, 0, 0, 0};
    for (const int end = min(hi, lo + length); lo < end; lo += VERIFY_BATCH, pt += VERIFY_BATCH, qt += Q ? VERIFY_BATCH : 0) {
      const int t = lo + lane;
      float x[N], y[N];
      if (lo + VERIFY_BATCH <= hi) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = __ldg(pt + 32 * e);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = Q ? __ldg(qt + 32 * e) : 0.f;
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const bool in = t + 32 * e < hi;
          x[e] = in ? __ldg(pt + 32 * e) : 0.f;
          y[e] = Q && in ? __ldg(qt + 32 * e) : 0.f;
        }
      }
      if (!Q) row.template mark<N>(y, lo, lane);
#pragma unroll
      for (int e = 0; e < N; ++e) s[e & 3] += row.weight(x[e], y[e]);
    }
    const double sum = warp_sum_d((s[0] + s[1]) + (s[2] + s[3]));
    if (lane == 0) seg[k] = sum;
    total += sum;
  }
  return total;
}

// The first of n parts that ends above the target, the last one with weight should rounding leave none; base: what lies before it.
__device__ __forceinline__ int part_of(const double *part, int n, double target, double &base) {
  int at = 0;
  double before = base;
  for (int i = 0; i < n; ++i) {
    const double s = part[i];
    if (!(s > 0)) continue;
    at = i;
    base = before;
    before += s;
    if (before > target) break;
  }
  return at;
}

struct DrawShared {
  double part[VERIFY_MAX_WARPS], seg[VERIFY_MAX_WARPS][32], all[2][VERIFY_MAX_CLUSTER];
};

// A cluster's look at one row of V entries.  Before its first total() every CTA arrives at the cluster's barrier (its shared memory is there).
struct ClusterRow {
  DrawShared &sh;
  cooperative_groups::cluster_group cluster;
  int C, c, lane, warp, warps, V, lo, hi, step, length, round;

  __device__ __forceinline__ ClusterRow(DrawShared &shared, int v) : sh(shared), cluster(cooperative_groups::this_cluster()), V(v), step(0), length(0), round(0) {
    C = (int)cluster.num_blocks(), c = (int)cluster.block_rank();
    lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    whole();
  }
  __device__ __forceinline__ void whole() {
    const int slice = (V + C - 1) / C;
    lo = min(V, c * slice), hi = min(V, lo + slice);
  }
  template <typename Row> __device__ __forceinline__ void level(const Row &row) {          // [lo, hi) by the CTA's warps
    const int each = ((hi - lo + warps - 1) / warps + VERIFY_BATCH - 1) / VERIFY_BATCH;
    step = each * VERIFY_BATCH;
    length = (each + 31) / 32 * VERIFY_BATCH;
    const int w0 = (int)min((long long)hi, lo + (long long)warp * step), w1 = (int)min((long long)hi, (long long)w0 + step);
    const double sum = row.q ? row_sums<true>(row, w0, w1, length, lane, sh.seg[warp]) : row_sums<false>(row, w0, w1, length, lane, sh.seg[warp]);
    if (lane == 0) sh.part[warp] = sum;
  }
  // All of the row's weight, for every thread of the cluster.
  template <typename Row> __device__ __forceinline__ double total(const Row &row) {
    double *const all = sh.all[round & 1];
    level(row);
    if (round++ == 0) cluster.barrier_wait();
    __syncthreads();
    if (warp == 0) {
      double s = 0;
      for (int i = 0; i < warps; ++i) s += sh.part[i];
      if (lane < C) *cluster.map_shared_rank(all + c, lane) = s;
    }
    cluster.sync();
    double sum = 0;
    for (int i = 0; i < C; ++i) sum += all[i];
    return sum;
  }
  // After total(): the smallest t whose running sum is above the target goes to *dst.
  template <typename Row> __device__ __forceinline__ void draw(const Row &row, double target, int *dst) {
    double base = 0;
    if (part_of(sh.all[(round - 1) & 1], C, target, base) != c) return;
#pragma unroll 1
    for (;;) {
      const int w = part_of(sh.part, warps, target, base);
      const int w0 = lo + w * step, w1 = min(hi, w0 + step);
      const int k = part_of(sh.seg[w], (w1 - w0 + length - 1) / length, target, base);
      lo = w0 + k * length;
      hi = min(w1, lo + length);
      if (length == VERIFY_BATCH) break;
      __syncthreads();
      level(row);
      __syncthreads();
    }
    if (warp == 0) {
      // eight entries a lane, in order
      constexpr int N = VERIFY_BATCH / 32;
      double x[N], s = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = lo + lane * N + e < hi ? row.at(lo + lane * N + e) : 0;
#pragma unroll
      for (int e = 0; e < N; ++e) s += x[e];
      double inc = s;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double v = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += v;
      }
      const unsigned over = __ballot_sync(0xffffffffu, s > 0 && base + inc > target), some = __ballot_sync(0xffffffffu, s > 0);
      if (lane == (over ? __ffs(over) - 1 : 31 - __clz(some))) {
        double cum = base + (inc - s);
        int drawn = -1;
        bool done = false;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          cum += x[e];
          if (x[e] > 0 && !done) drawn = lo + lane * N + e, done = cum > target;
        }
        *dst = drawn;
      }
    }
  }
};

}  // namespace tsfm
