// Verification of a tree of drafted tokens against the target's probabilities (tsfm_verify_tree): the accepted path, and the token drawn
// behind it.
#pragma once
#include "draw_row.cuh"
#include "tree.cuh"

namespace tsfm {

struct VerifyTreeArgs {
  const int *tokens, *parent;
  long long parent_series;                         // from a series to the next: 0 with one tree for all
  const float *p, *q;                              // q or NULL
  long long p_stride, q_stride;
  int M, V;
  const float *u;                                  // or NULL: Philox
  uint2 key;
  int round_idx, series0;
  const int *n_new, *len;                          // or NULL
  int *out, *path, *n_accept, *len_out;
};

// What is left of node c's row once some of its children were rejected: max(p - used q, 0), or without a distribution p without those
// children's tokens.  (With r_0 = p, Z_0 = 1 the rest after a rejection is r_k+1 = max(r_k - Z_k q, 0): as q >= 0, that is
// max(p - (Z_0 + .. + Z_k) q, 0), so `used` alone describes it.)
struct TreeRow {
  const float *p, *q;                              // q or NULL
  double used;
  const int *gone;                                 // shared memory: tokens without weight
  int n_gone;
  __device__ __forceinline__ double weight(float x, float y) const {
    const double w = draw_weight(x);
    return q ? w - fmin(w, used * (double)draw_weight(y)) : y != 0.f ? 0. : w;
  }
  __device__ __forceinline__ bool is_gone(int t) const {
    bool hit = false;
    for (int i = 0; i < n_gone; ++i) hit |= gone[i] == t;
    return hit;
  }
  // y != 0: gone.  The lanes look for rejected tokens among the batch's 256 entries together; mostly there are none.
  template <int N> __device__ __forceinline__ void mark(float (&y)[N], int lo, int lane) const {
    bool some = false;
    for (int i = lane; i < n_gone; i += 32) some |= (unsigned)(gone[i] - lo) < (unsigned)VERIFY_BATCH;
    if (!__any_sync(0xffffffffu, some)) return;
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = is_gone(lo + lane + 32 * e) ? 1.f : 0.f;
  }
  __device__ __forceinline__ double at(int t) const { return weight(__ldg(p + t), q ? __ldg(q + t) : is_gone(t) ? 1.f : 0.f); }
};

// A cluster of CTAs a series (draw_row.cuh).  All nodes' probabilities are gathered first, at once: the walk then reads shared memory, every
// warp takes it by itself and arrives at the same nodes.  A rejection whose node has another child asks for the sum of what is left, one
// look of the cluster at the two rows; the last row is summed for the draw.
// Bound: the chain of looks (64 trees of 33 nodes, 100003 tokens: 41 us, of which two rows from memory are 8).
__global__ void __launch_bounds__(32 * VERIFY_MAX_WARPS, 2) verify_tree_kernel(VerifyTreeArgs a) {
  __shared__ DrawShared sh;
  __shared__ int parent_s[TREE_MAX], token_s[TREE_MAX], path_s[TREE_MAX], gone_s[TREE_MAX], n_gone;
  __shared__ float px_s[TREE_MAX], qx_s[TREE_MAX], u_s[TREE_MAX + 1];
  cooperative_groups::this_cluster().barrier_arrive();        // (waited for before the first store to another CTA's shared memory)
  ClusterRow look(sh, a.V);
  const int b = blockIdx.x / look.C, lane = look.lane, M = a.M, V = a.V, tid = threadIdx.x;
  const int nodes = a.n_new ? min(max(a.n_new[b], 0), M) : M;
  const float *p0 = a.p + (long long)b * M * a.p_stride, *q0 = a.q ? a.q + (long long)b * M * a.q_stride : nullptr;
  int *const out = a.out + (long long)b * M, *const path = a.path + (long long)b * M;
  auto uniform = [&](int i) {
    return a.u ? a.u[(long long)b * (M + 1) + i]
               : uniform_from_word(philox4x32_10(make_uint4((uint32_t)(a.series0 + b), (uint32_t)a.round_idx, (uint32_t)i, 0u), a.key).x);
  };
  if (tid == 0) n_gone = 0, u_s[M] = uniform(M);
  for (int m = tid; m < nodes; m += blockDim.x) {
    const int up = m ? a.parent[b * a.parent_series + m] : -1, x = a.tokens[(long long)b * M + m];
    float px = 0.f, qx = 1.f;
    if (up >= 0 && up < m && (unsigned)x < (unsigned)V) {
      px = draw_weight(p0[up * a.p_stride + x]);
      if (q0) qx = draw_weight(q0[up * a.q_stride + x]);
    }
    parent_s[m] = up < m ? up : -1;
    token_s[m] = x;
    px_s[m] = px;
    qx_s[m] = qx;
    u_s[m] = uniform(m);
  }
  __syncthreads();
  if (nodes == 0) {                                // (a padded series; the whole cluster leaves)
    look.cluster.barrier_wait();
    if (look.c == 0) {
      for (int i = tid; i < M; i += blockDim.x) out[i] = path[i] = -1;
      if (tid == 0) {
        a.n_accept[b] = 0;
        if (a.len_out) a.len_out[b] = a.len[b];
      }
    }
    return;
  }
  int here = 0, tried = 0, n = 0;
  double used = 0, mass = 1;
  auto next_child = [&]() {                        // of `here`, behind `tried`; -1: none
    for (int at = tried & ~31; at < nodes; at += 32) {
      const int i = at + lane;
      const unsigned is = __ballot_sync(0xffffffffu, i > tried && i < nodes && parent_s[min(i, nodes - 1)] == here);
      if (is) return at + __ffs(is) - 1;
    }
    return -1;
  };
  if (tid == 0) path_s[0] = 0;
#pragma unroll 1
  for (int child = next_child(); child >= 0;) {
    double px = px_s[child];
    const double qx = qx_s[child];
    if (!q0) {                                     // (picked twice: its weight is gone)
      bool again = false;
      for (int i = lane; i < child; i += 32) again |= parent_s[i] == here && i <= tried && i > here && token_s[i] == token_s[child];
      if (__any_sync(0xffffffffu, again)) px = 0;
    }
    const double rest = q0 ? px - fmin(px, used * qx) : px;
    tried = child;
    if (draw_uniform(u_s[child]) * qx * mass < rest) {
      here = child;
      ++n;
      if (tid == 0) path_s[n] = child;
      used = 0, mass = 1;
      child = next_child();
    } else {
      child = next_child();
      if (!q0) {
        mass -= px;
      } else {
        used += mass;
        if (child >= 0) mass = look.total(TreeRow{p0 + here * a.p_stride, q0 + here * a.q_stride, used, gone_s, 0});
      }
    }
  }
  if (!q0)
    for (int i = tid; i < nodes; i += blockDim.x)
      if (i > here && i <= tried && parent_s[i] == here) gone_s[atomicAdd(&n_gone, 1)] = token_s[i];
  __syncthreads();
  TreeRow row{p0 + here * a.p_stride, used > 0 ? q0 + here * a.q_stride : nullptr, used, gone_s, n_gone};
#pragma unroll 1
  for (int attempt = 0; attempt < 2; ++attempt) {
    const double total = look.total(row);
    if (total > 0) {
      look.draw(row, draw_uniform(u_s[M]) * total, out + n);
      break;
    }
    if (attempt == 1) {
      if (look.c == 0 && tid == 0) out[n] = -1;
      break;
    }
    row.q = nullptr;                               // nothing is left: draw from p
    row.n_gone = 0;
  }
  if (look.c) return;
  for (int i = tid; i < M; i += blockDim.x) {
    if (i != n) out[i] = i < n ? token_s[path_s[i + 1]] : -1;
    path[i] = i <= n ? path_s[i] : -1;
  }
  if (tid == 0) {
    a.n_accept[b] = n;
    if (a.len_out) a.len_out[b] = a.len[b] + n + 1;
  }
}

}  // namespace tsfm
