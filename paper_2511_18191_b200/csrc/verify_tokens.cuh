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

constexpr int VERIFY_MAX_WARPS = 16, VERIFY_MAX_CLUSTER = 8, VERIFY_BATCH = 256;

// A probability as a weight of the draw: what is negative or not finite counts as 0.  (The bits of a positive finite float are
// 1 .. 0x7f7fffff.)
__device__ __forceinline__ float draw_weight(float p) { return __float_as_uint(p) - 1u < 0x7f7fffffu ? p : 0.f; }

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
  // Sums over [lo, hi) by a warp, one of every `length` entries (a multiple of 256) into seg[], and all of them, in all lanes.
  // Sixteen loads of a lane in flight (eight without q): with what the compiler had gathered by itself the batch of 256 rows of 100003 took 132 us.
  __device__ __forceinline__ double sums(int lo, int hi, int length, int lane, double *seg) const {
    return q ? sums_of<true>(lo, hi, length, lane, seg) : sums_of<false>(lo, hi, length, lane, seg);
  }
  template <bool Q> __device__ __forceinline__ double sums_of(int lo, int hi, int length, int lane, double *seg) const {
    constexpr int N = VERIFY_BATCH / 32;
    double total = 0;
    const float *pt = p + lo + lane, *qt = Q ? q + lo + lane : nullptr;
    for (int k = 0; lo < hi; ++k) {
      double s[4] = {0, 0, 0, 0};
      for (const int end = min(hi, lo + length); lo < end; lo += VERIFY_BATCH, pt += VERIFY_BATCH, qt += Q ? VERIFY_BATCH : 0) {
        const int t = lo + lane;
        float x[N], y[N];
        if (lo + VERIFY_BATCH <= hi) {
#pragma unroll
          for (int e = 0; e < N; ++e) x[e] = __ldg(pt + 32 * e);
#pragma unroll
          for (int e = 0; e < N; ++e) y[e] = Q ? __ldg(qt + 32 * e) : t + 32 * e == without ? 1.f : 0.f;
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const bool in = t + 32 * e < hi;
            x[e] = in ? __ldg(pt + 32 * e) : 0.f;
            y[e] = Q ? (in ? __ldg(qt + 32 * e) : 0.f) : t + 32 * e == without ? 1.f : 0.f;
          }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) s[e & 3] += rest(x[e], y[e]);
      }
      const double sum = warp_sum_d((s[0] + s[1]) + (s[2] + s[3]));
      if (lane == 0) seg[k] = sum;
      total += sum;
    }
    return total;
  }
};

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

// A cluster of CTAs a series; CTA c, and in it each warp, sums a contiguous part of the row, and keeps the sums of up to 32
// segments of it.  The draw then falls into a CTA's, a warp's, a segment's part: 256 entries for rows of up to 32 x 256 a warp, which one
// warp looks through; a longer segment is shared by the CTA's warps as the row was.  Sums are fp64 so that their order decides nothing.
// Bound: memory, behind the chain proposals - their probabilities - row (256 rows of 100003, 0.8 of the proposals accepted: 43 us, 4.0 TB/s; without q
// 47 after a flush of L2: half the bytes, the same chain).  (In place of the segments' sums three more passes over ever
// smaller parts cost 10 us.)
__global__ void __launch_bounds__(32 * VERIFY_MAX_WARPS, 2) verify_tokens_kernel(VerifyArgs a) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ double part[VERIFY_MAX_WARPS], seg[VERIFY_MAX_WARPS][32], all[2][VERIFY_MAX_CLUSTER];
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
  const int slice = (V + C - 1) / C;
  int lo = min(V, c * slice), hi = min(V, lo + slice), step = 0, length = 0;
  auto level = [&]() {                             // [lo, hi) by the CTA's warps
    const int each = ((hi - lo + warps - 1) / warps + VERIFY_BATCH - 1) / VERIFY_BATCH;
    step = each * VERIFY_BATCH;
    length = (each + 31) / 32 * VERIFY_BATCH;
    const int w0 = (int)min((long long)hi, lo + (long long)warp * step), w1 = (int)min((long long)hi, (long long)w0 + step);
    const double sum = row.sums(w0, w1, length, lane, seg[warp]);
    if (lane == 0) part[warp] = sum;
  };
#pragma unroll 1
  for (int attempt = 0; attempt < 2; ++attempt) {
    level();
    if (attempt == 0) cluster.barrier_wait();
    __syncthreads();
    if (warp == 0) {
      double s = 0;
      for (int i = 0; i < warps; ++i) s += part[i];
      if (lane < C) *cluster.map_shared_rank(&all[attempt][c], lane) = s;
    }
    cluster.sync();
    double total = 0;
    for (int i = 0; i < C; ++i) total += all[attempt][i];
    if (total > 0) {
      const double target = (double)fminf(fmaxf(uniform(K), 0.f), 0.999999940395355224609375f) * total;
      double base = 0;
      if (part_of(all[attempt], C, target, base) != c) break;
#pragma unroll 1
      for (;;) {
        const int w = part_of(part, warps, target, base);
        const int w0 = lo + w * step, w1 = min(hi, w0 + step);
        const int k = part_of(seg[w], (w1 - w0 + length - 1) / length, target, base);
        lo = w0 + k * length;
        hi = min(w1, lo + length);
        if (length == VERIFY_BATCH) break;
        __syncthreads();
        level();
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
          a.out[(long long)b * (K + 1) + n] = drawn;
        }
      }
      break;
    }
    if (attempt == 1) {
      if (c == 0 && threadIdx.x == 0) a.out[(long long)b * (K + 1) + n] = -1;
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
