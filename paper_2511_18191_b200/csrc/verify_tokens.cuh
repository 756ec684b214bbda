// Verification of drafted tokens against the target's probabilities (tsfm_verify_tokens): the first rejection, and the token
// drawn in its place, by inverse CDF.
#pragma once
#include <cooperative_groups.h>
#include "accept.cuh"

namespace tsfm {

struct VerifyArgs {
  const int *tokens;
  const float *p, *q;                              // q or NULL
  long long p_stride, q_stride;
  int K, V;
  const float *u;                                  // or NULL: Philox
  uint2 key;
  int round_idx, series0;
  const int *n_draft, *len;                        // or NULL
  int *out, *n_accept, *len_out;
};

// A probability as a weight of the draw: what is negative or not finite counts as 0.
__device__ __forceinline__ float draw_weight(float p) { return p > 0.f && p < INFINITY ? p : 0.f; }

// What a token is drawn from: max(p - q, 0) for a row q, p without one token (q is 1 there), or p.
struct DrawRow {
  const float *p, *q;                              // q or NULL
  int without;                                     // or -1
  __device__ __forceinline__ float p_at(int t) const { return __ldg(p + t); }
  __device__ __forceinline__ float q_at(int t) const { return q ? __ldg(q + t) : t == without ? 1.f : 0.f; }
  static __device__ __forceinline__ double rest(float p, float q) {
    const float x = draw_weight(p);
    return (double)x - (double)fminf(x, draw_weight(q));
  }
  __device__ __forceinline__ double at(int t) const { return rest(p_at(t), q_at(t)); }
  // The sum over [lo, hi) by a warp, in all lanes.  Sixteen loads of a lane in flight: with what the compiler had gathered by
  // itself the batch of 256 rows of 100003 took 132 us.
  __device__ __forceinline__ double sum(int lo, int hi, int lane) const { return q ? sum_of<true>(lo, hi, lane) : sum_of<false>(lo, hi, lane); }
  template <bool Q> __device__ __forceinline__ double sum_of(int lo, int hi, int lane) const {
    constexpr int N = 8;
    double s[4] = {0, 0, 0, 0};
    for (int t0 = lo + lane; t0 < hi; t0 += 32 * N) {
      float x[N], y[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int t = t0 + 32 * e;
        x[e] = t < hi ? p_at(t) : 0.f;
        y[e] = Q ? (t < hi ? __ldg(q + t) : 0.f) : t == without ? 1.f : 0.f;
      }
#pragma unroll
      for (int e = 0; e < N; ++e) s[e & 3] += rest(x[e], y[e]);
    }
    return warp_sum_d((s[0] + s[1]) + (s[2] + s[3]));
  }
};

// A cluster of CTAs a series; CTA c, and in it each warp, sums a contiguous part of the row.  Everything after the sums
// happens in the CTA, then the warp, whose part the draw falls into.  Sums are fp64 so that their order decides nothing.
constexpr int VERIFY_MAX_WARPS = 16, VERIFY_MAX_CLUSTER = 8, VERIFY_LAST = 512;
__global__ void __launch_bounds__(32 * VERIFY_MAX_WARPS) verify_tokens_kernel(VerifyArgs a) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ double part[VERIFY_MAX_WARPS], all[2][VERIFY_MAX_CLUSTER];
  __shared__ int first_bad;
  cluster.barrier_arrive();                        // (waited for before the first store to another CTA's shared memory)
  const int C = (int)cluster.num_blocks(), c = (int)cluster.block_rank(), b = blockIdx.x / C;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, K = a.K, V = a.V;
  const int nd = a.n_draft ? min(max(a.n_draft[b], 0), K) : K;
  const float *p0 = a.p + (long long)b * (K + 1) * a.p_stride, *q0 = a.q ? a.q + (long long)b * K * a.q_stride : nullptr;
  auto uniform = [&](int i) {
    return a.u ? a.u[(long long)b * (K + 1) + i]
               : uniform_from_word(philox4x32_10(make_uint4((uint32_t)(a.series0 + b), (uint32_t)a.round_idx, (uint32_t)i, 0u), a.key).x);
  };
  if (warp == 0) {
    bool ok = true;
    if (lane < nd) {
      const int x = a.tokens[(long long)b * K + lane];
      ok = false;
      if ((unsigned)x < (unsigned)V) {
        const double px = draw_weight(p0[lane * a.p_stride + x]), qx = q0 ? draw_weight(q0[lane * a.q_stride + x]) : 1.f;
        const float u = uniform(lane);
        ok = (double)fminf(fmaxf(u, 0.f), 0.999999940395355224609375f) * qx < px;     // 24 bits by 24 bits: exact
      }
    }
    const unsigned rejected = __ballot_sync(0xffffffffu, !ok);
    if (lane == 0) first_bad = rejected ? __ffs(rejected) - 1 : nd;
  }
  __syncthreads();
  const int n = first_bad;
  DrawRow row{p0 + n * a.p_stride, n < nd && q0 ? q0 + n * a.q_stride : nullptr, n < nd && !q0 ? a.tokens[(long long)b * K + n] : -1};
  const int slice = (V + C - 1) / C, v0 = min(V, c * slice), v1 = min(V, v0 + slice);
  const int step = (slice + warps - 1) / warps;
  const int w0 = min(v1, v0 + warp * step), w1 = min(v1, w0 + step);
  double total = 0, mine = 0;
#pragma unroll 1
  for (int attempt = 0; attempt < 2; ++attempt) {
    mine = row.sum(w0, w1, lane);
    if (lane == 0) part[warp] = mine;
    if (attempt == 0) cluster.barrier_wait();
    __syncthreads();
    if (warp == 0) {
      double s = 0;
      for (int i = 0; i < warps; ++i) s += part[i];
      if (lane < C) *cluster.map_shared_rank(&all[attempt][c], lane) = s;
    }
    cluster.sync();
    total = 0;
    for (int i = 0; i < C; ++i) total += all[attempt][i];
    if (total > 0 || attempt == 1) {
      double before = 0, target = 0;
      const float u = uniform(K);
      target = (double)fminf(fmaxf(u, 0.f), 0.999999940395355224609375f) * total;
      // the CTA whose part holds the target (the last one with weight, should rounding leave none)
      int owner = -1;
      double base = 0;
      for (int i = 0; i < C; ++i) {
        const double s = all[attempt][i];
        if (!(s > 0)) continue;
        owner = i;
        base = before;
        before += s;
        if (before > target) break;
      }
      int drawn = -1;
      if (owner == c) {
        // the warp's part, then ever smaller parts shared by the CTA's warps, until one warp can take the rest
        int lo = v0, width = step, end = v1;
#pragma unroll 1
        for (;;) {
          int at = -1;
          double sum = base, start = base;
          for (int i = 0; i < warps; ++i) {
            const double s = part[i];
            if (!(s > 0)) continue;
            at = i;
            start = sum;
            sum += s;
            if (sum > target) break;
          }
          base = start;
          lo += max(at, 0) * width;
          end = min(end, lo + width);
          if (width <= VERIFY_LAST) break;
          width = (width + warps - 1) / warps;
          const int x0 = min(end, lo + warp * width), x1 = min(end, x0 + width);
          const double s = row.sum(x0, x1, lane);
          __syncthreads();
          if (lane == 0) part[warp] = s;
          __syncthreads();
        }
        if (warp == 0) {
          // a contiguous run of entries a lane
          const int run = (end - lo + 31) / 32;
          double s = 0;
          for (int i = 0; i < run; ++i) {
            const int t = lo + lane * run + i;
            if (t < end) s += row.at(t);
          }
          double inc = s;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const double v = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += v;
          }
          const unsigned over = __ballot_sync(0xffffffffu, s > 0 && base + inc > target), some = __ballot_sync(0xffffffffu, s > 0);
          const int who = over ? __ffs(over) - 1 : some ? 31 - __clz(some) : -1;
          if (lane == who) {
            double cum = base + (inc - s);
            for (int i = 0; i < run; ++i) {
              const int t = lo + lane * run + i;
              if (t >= end) break;
              const double x = row.at(t);
              cum += x;
              if (x > 0) drawn = t;
              if (x > 0 && cum > target) break;
            }
            a.out[(long long)b * (K + 1) + n] = drawn;
          }
          if (who < 0 && lane == 0) a.out[(long long)b * (K + 1) + n] = -1;
        }
      } else if (owner < 0 && c == 0 && threadIdx.x == 0) {
        a.out[(long long)b * (K + 1) + n] = -1;
      }
      break;
    }
    row.q = nullptr;                               // p nowhere above q: draw from p
    row.without = -1;
  }
  if (c == 0 && threadIdx.x <= K && (int)threadIdx.x != n)
    a.out[(long long)b * (K + 1) + threadIdx.x] = (int)threadIdx.x < n ? a.tokens[(long long)b * K + threadIdx.x] : -1;
  if (c == 0 && threadIdx.x == 0) {
    a.n_accept[b] = n;
    if (a.len_out) a.len_out[b] = a.len[b] + n + 1;
  }
}

}  // namespace tsfm
