// Trees of drafted tokens: what their nodes see (tsfm_tree_init), and the accepted path's move to the front of the cache
// (tsfm_cache_commit).
#pragma once
#include "pages.cuh"

namespace tsfm {

constexpr int TREE_MAX = 256;                      // TSFM_MAX_TREE

// A CTA a tree, a thread a node, which walks up to its root.  Bound: launch; a walk is a chain of reads of shared memory as long as the node is
// deep.
__global__ void __launch_bounds__(TREE_MAX) tree_init_kernel(const int *parent, const int *n_new, int M, int words, int window, unsigned long long *mask, int *depth) {
  __shared__ int up[TREE_MAX];
  __shared__ unsigned long long bits[TREE_MAX][TREE_MAX / 64];
  const int b = blockIdx.x, m = threadIdx.x;
  const int nodes = n_new ? cut(n_new[b], M) : M;
  if (m < M) {
    const int p = parent[(long long)b * M + m];
    up[m] = p >= 0 && p < m ? p : -1;
  }
  for (int w = 0; w < TREE_MAX / 64; ++w) bits[m][w] = 0;
  __syncthreads();
  if (m >= M) return;
  int above = 0;
  if (m < nodes) {
    for (int i = m; i >= 0; i = up[i], ++above)
      if (!window || above < window) bits[m][i >> 6] |= 1ull << (i & 63);
    --above;
  }
  for (int w = 0; w < words; ++w) mask[((long long)b * M + m) * words + w] = bits[m][w];
  depth[(long long)b * M + m] = above;
}

struct CommitArgs {
  PagesDev pg;
  const int *path, *len;
  long long layer_stride;                          // bytes
  int B, M, n_layers, vecs, blocks;                // vecs: 16-byte vectors of a row; blocks: CTAs of a series
};

// A thread moves one 16-byte column of one head, layer and of keys or values along the path, eight slots at a time.  The path ascends, so a slot
// is written only once what it held has been read: path[i] >= i, and the eight loads of a turn stand before its stores.
// Bound: latency (path -> pages -> rows), then memory (24 layers x 64 series, up to 8 tokens of 8 heads of 128: 13 to 15 us, 46 MB).
constexpr int COMMIT_THREADS = 256;
__global__ void __launch_bounds__(COMMIT_THREADS) cache_commit_kernel(const __grid_constant__ CommitArgs a) {
  __shared__ long long from_s[TREE_MAX], to_s[TREE_MAX];
  __shared__ int steps_s, first_bad;
  const int b = blockIdx.x / a.blocks, part = blockIdx.x - b * a.blocks, tid = threadIdx.x;
  const int *path = a.path + (long long)b * a.M;
  if (tid == 0) steps_s = 0, first_bad = a.M;
  __syncthreads();
  const int mine = tid < a.M ? path[tid] : -1;
  if (tid < a.M && (mine < 0 || mine >= a.M || (tid && mine <= path[tid - 1]))) atomicMin(&first_bad, tid);
  __syncthreads();
  if (tid < first_bad && mine != tid) {            // (behind the first node that moves every one does: the order stays)
    const long long len = a.len[b], from = len + mine, to = len + tid;
    long long src = -1, dst = -1;
    if (to >= 0 && from < a.pg.capacity) {
      const int *row = a.pg.table + (long long)b * a.pg.table_stride;
      const int p = page_of(a.pg, row, (int)from), q = page_of(a.pg, row, (int)to);
      if (p < 0 || q < 0) pages_report(a.pg, BAD_ID);
      else src = slot_offset(a.pg, p, 0, (int)from), dst = slot_offset(a.pg, q, 0, (int)to);
    } else {
      pages_report(a.pg, BAD_LEN);
    }
    from_s[tid] = src;
    to_s[tid] = dst;
    atomicMax(&steps_s, tid + 1);
  } else if (tid < a.M) {
    from_s[tid] = to_s[tid] = -1;
  }
  __syncthreads();
  const int steps = steps_s;
  if (!steps) return;
  const long long items = (long long)a.n_layers * a.pg.n_kv_heads * 2 * a.vecs;
  for (long long i = (long long)part * COMMIT_THREADS + tid; i < items; i += (long long)a.blocks * COMMIT_THREADS) {
    const long long rest = i / a.vecs;
    const int vec = (int)(i - rest * a.vecs), kv = (int)(rest & 1), h = (int)((rest >> 1) % a.pg.n_kv_heads), layer = (int)((rest >> 1) / a.pg.n_kv_heads);
    char *base = (kv ? a.pg.v : a.pg.k) + layer * a.layer_stride + h * a.pg.head_stride + vec * 16;
    for (int s0 = 0; s0 < steps; s0 += 8) {
      uint4 x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (s0 + j < steps && from_s[s0 + j] >= 0) x[j] = *reinterpret_cast<const uint4 *>(base + from_s[s0 + j]);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (s0 + j < steps && from_s[s0 + j] >= 0) *reinterpret_cast<uint4 *>(base + to_s[s0 + j]) = x[j];
    }
  }
}

}  // namespace tsfm
