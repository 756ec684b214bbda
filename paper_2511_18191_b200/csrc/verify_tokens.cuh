// Verification of drafted tokens against the target's probabilities (tsfm_verify_tokens): the first rejection, and the token
// drawn in its place.
#pragma once
#include "draw_row.cuh"

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

// What a token is drawn from: max(p - q, 0) for a row q, p without one token (q is 1 there), or p.
struct DrawRow {
  const float *p, *q;                              // q or NULL
  int without;                                     // or -1
  static __device__ __forceinline__ double weight(float p, float q) {
    const float x = draw_weight(p);
    return (double)x - (double)fminf(x, draw_weight(q));
  }
  template <int N> __device__ __forceinline__ void mark(float (&y)[N], int lo, int lane) const {
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = lo + lane + 32 * e == without ? 1.f : 0.f;
  }
  __device__ __forceinline__ double at(int t) const { return weight(__ldg(p + t), q ? __ldg(q + t) : t == without ? 1.f : 0.f); }
};

// A cluster of CTAs a series (draw_row.cuh).  Bound: memory, behind the chain proposals - their probabilities - row (256 rows of 100003, 0.8 of
// the proposals accepted: 43 us, 4.0 TB/s; without q 47 after a flush of L2: half the bytes, the same chain).  (In place of the segments' sums
// three more passes over ever smaller parts cost 10 us.)
__global__ void __launch_bounds__(32 * VERIFY_MAX_WARPS, 2) verify_tokens_kernel(VerifyArgs a) {
  __shared__ DrawShared sh;
  __shared__ int first_bad;
  cooperative_groups::this_cluster().barrier_arrive();        // (waited for before the first store to another CTA's shared memory)
  ClusterRow look(sh, a.V);
  const int b = blockIdx.x / look.C, lane = look.lane, K = a.K, V = a.V;
  const int nd = a.n_draft ? min(max(a.n_draft[b], 0), K) : K;
  const float *p0 = a.p + (long long)b * (K + 1) * a.p_stride, *q0 = a.q ? a.q + (long long)b * K * a.q_stride : nullptr;
  auto uniform = [&](int i) {
    return a.u ? a.u[(long long)b * (K + 1) + i]
               : uniform_from_word(philox4x32_10(make_uint4((uint32_t)(a.series0 + b), (uint32_t)a.round_idx, (uint32_t)i, 0u), a.key).x);
  };
  if (look.warp == 0) {
    bool ok = true;
    if (lane < nd) {
      const int x = a.tokens[(long long)b * K + lane];
      ok = false;
      if ((unsigned)x < (unsigned)V) {
        const double px = draw_weight(p0[lane * a.p_stride + x]), qx = q0 ? draw_weight(q0[lane * a.q_stride + x]) : 1.f;
        ok = draw_uniform(uniform(lane)) * qx < px;           // 24 bits by 24 bits: exact
      }
    }
    const unsigned rejected = __ballot_sync(0xffffffffu, !ok);
    if (lane == 0) first_bad = rejected ? __ffs(rejected) - 1 : nd;
  }
  __syncthreads();
  const int n = first_bad;
  int *const dst = a.out + (long long)b * (K + 1) + n;
  DrawRow row{p0 + n * a.p_stride, n < nd && q0 ? q0 + n * a.q_stride : nullptr, n < nd && !q0 ? a.tokens[(long long)b * K + n] : -1};
#pragma unroll 1
  for (int attempt = 0; attempt < 2; ++attempt) {
    const double total = look.total(row);
    if (total > 0) {
      look.draw(row, draw_uniform(uniform(K)) * total, dst);
      break;
    }
    if (attempt == 1) {
      if (look.c == 0 && threadIdx.x == 0) *dst = -1;
      break;
    }
    row.q = nullptr;                               // p nowhere above q: draw from p
    row.without = -1;
  }
  if (look.c == 0 && threadIdx.x <= K && (int)threadIdx.x != n)
    a.out[(long long)b * (K + 1) + threadIdx.x] = (int)threadIdx.x < n ? a.tokens[(long long)b * K + threadIdx.x] : -1;
  if (look.c == 0 && threadIdx.x == 0) {
    a.n_accept[b] = n;
    if (a.len_out) a.len_out[b] = a.len[b] + n + 1;
  }
}

}  // namespace tsfm
