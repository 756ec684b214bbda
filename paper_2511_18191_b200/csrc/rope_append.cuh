// Rotary positions of new tokens and the append to a cache of pages (tsfm_rope_append): one pass over the tokens' stacked
// query, key and value rows, queries out, keys and values into their slots.
#pragma once
#include "pages.cuh"

namespace tsfm {

constexpr int ROPE_MAX_PAIRS = 64;
struct RopeAppendArgs {
  PagesDev pg;
  const void *qkv;
  void *q_out;                                     // or NULL
  long long qkv_stride, q_stride;                  // elements
  const int *pos, *len, *n_new;                    // pos, n_new or NULL
  int tokens, M, n_heads, half;                    // half: 1 pairs (i, i + rot / 2), 0 pairs (2 i, 2 i + 1)
  int pairs;                                       // rot / 2
  int head_lanes, token_lanes;                     // heads and tokens that a CTA works on at once
  float mscale;
  uint64_t turn[ROPE_MAX_PAIRS];                   // 2^64 x turns a position
};

// cos and sin of position t: the angle in turns is the low 64 bits of t * turn, exact modulo a whole turn, so that far
// positions lose nothing; 32 of them go into the float.
__device__ __forceinline__ float2 rope_cos_sin(uint64_t turn, long long t, float mscale) {
  const uint64_t phase = turn * (uint64_t)t;
  float s, c;
  sincospif((float)(int)(phase >> 32) * 4.656612873077392578125e-10f, &s, &c);      // 2^-31: half turns
  return make_float2(c * mscale, s * mscale);
}

// A unit is what a thread turns at once in a head: with `half` a vector of the first half and its partner (or a vector
// behind the turned part), interleaved a vector.  A thread keeps its unit and goes over the token's heads, so that the
// angles of a unit are read once; the first two heads are on their way while the angles are computed.
template <typename T, bool HALF>
__global__ void __launch_bounds__(256) rope_append_kernel(const __grid_constant__ RopeAppendArgs a, int D) {
  constexpr int V = Pack16<T>::N, N = 2;           // heads in flight
  extern __shared__ float2 cs[];                                 // [token lane][pair]
  const int vecs = D / V, half_vecs = a.pairs / V;
  const int units = HALF ? vecs - half_vecs : vecs;
  const int u = threadIdx.x % units, rest = threadIdx.x / units;
  const int hl = rest % a.head_lanes, tl = rest / a.head_lanes;
  const int Hkv = a.pg.n_kv_heads, heads = a.n_heads + 2 * Hkv;
  const int t0 = blockIdx.x * a.token_lanes, tok = t0 + tl;
  const int first = HALF && u >= half_vecs ? u + half_vecs : u;  // this unit's vectors of a head
  const bool pair = HALF && u < half_vecs;
  const int second = first + half_vecs;
  const bool mine = tl < a.token_lanes && tok < a.tokens;
  const int b = mine ? tok / a.M : 0, m = tok - b * a.M;
  const T *src = reinterpret_cast<const T *>(a.qkv) + (long long)(mine ? tok : 0) * a.qkv_stride;
  Pack16<T> x[N], y[N];
  auto fetch = [&](int h) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const T *s = src + (h + j * a.head_lanes) * D;
      if (mine && h + j * a.head_lanes < heads) {
        x[j].raw = *reinterpret_cast<const uint4 *>(s + first * V);
        if (pair) y[j].raw = *reinterpret_cast<const uint4 *>(s + second * V);
      }
    }
  };
  int h = (a.q_out ? 0 : a.n_heads) + hl;
  fetch(h);
  for (int i = threadIdx.x; i < a.token_lanes * a.pairs; i += blockDim.x) {
    const int at = i / a.pairs, p = i - at * a.pairs, t = t0 + at;
    if (t < a.tokens) {
      const int tb = t / a.M;
      cs[i] = rope_cos_sin(a.turn[p], (long long)(a.pos ? a.pos[tb] : a.len[tb]) + t - tb * a.M, a.mscale);
    }
  }
  const bool live = mine && (!a.n_new || m < a.n_new[b]);
  // the token's slot
  const long long slot = mine ? (long long)a.len[b] + m : 0;
  int page = -1;
  if (live) {
    const bool in = slot >= 0 && slot < a.pg.capacity;
    if (in) page = page_of(a.pg, a.pg.table + (long long)b * a.pg.table_stride, (int)slot);
    if (page < 0 && u == 0 && hl == 0) pages_report(a.pg, in ? BAD_ID : BAD_LEN);
  }
  __syncthreads();
  if (!live) return;
  const float2 *ang = cs + tl * a.pairs;
  T *qdst = a.q_out ? reinterpret_cast<T *>(a.q_out) + (long long)tok * a.q_stride : nullptr;
  for (; h < heads; fetch(h += N * a.head_lanes)) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int hj = h + j * a.head_lanes;
      if (hj >= heads) break;
      if (hj < a.n_heads + Hkv) {
        if (pair) {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float2 c = ang[u * V + e];
            const float p = x[j].get(e), q = y[j].get(e);
            x[j].set(e, p * c.x - q * c.y);
            y[j].set(e, q * c.x + p * c.y);
          }
        } else if (!HALF) {
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            if (u * V + e < 2 * a.pairs) {
              const float2 c = ang[(u * V + e) >> 1];
              const float p = x[j].get(e), q = x[j].get(e + 1);
              x[j].set(e, p * c.x - q * c.y);
              x[j].set(e + 1, q * c.x + p * c.y);
            }
          }
        }
      }
      T *d;
      if (hj < a.n_heads) {
        d = qdst + hj * D;
      } else {
        if (page < 0) continue;
        const bool key = hj < a.n_heads + Hkv;
        d = reinterpret_cast<T *>((key ? a.pg.k : a.pg.v) + slot_offset(a.pg, page, hj - a.n_heads - (key ? 0 : Hkv), (int)slot));
      }
      *reinterpret_cast<uint4 *>(d + first * V) = x[j].raw;
      if (pair) *reinterpret_cast<uint4 *>(d + second * V) = y[j].raw;
    }
  }
}

// HALF with a half that is no whole number of vectors: element pairs (and the single elements behind the turned part), one
// a thread.  A thread reads both elements of a pair before it writes them, so in place works here too.
template <typename T>
__global__ void __launch_bounds__(256) rope_append_odd_kernel(const __grid_constant__ RopeAppendArgs a, int D) {
  __shared__ float2 cs[ROPE_MAX_PAIRS];
  const int tok = blockIdx.x, b = tok / a.M, m = tok - b * a.M;
  if (a.n_new && m >= a.n_new[b]) return;
  if (threadIdx.x < a.pairs) cs[threadIdx.x] = rope_cos_sin(a.turn[threadIdx.x], (long long)(a.pos ? a.pos[b] : a.len[b]) + m, a.mscale);
  __syncthreads();
  const long long slot = (long long)a.len[b] + m;
  int page = -1;
  if (slot < 0 || slot >= a.pg.capacity) {
    if (threadIdx.x == 0) pages_report(a.pg, BAD_LEN);
  } else {
    page = page_of(a.pg, a.pg.table + (long long)b * a.pg.table_stride, (int)slot);
    if (page < 0 && threadIdx.x == 0) pages_report(a.pg, BAD_ID);
  }
  const int Hkv = a.pg.n_kv_heads, heads = a.n_heads + 2 * Hkv, units = D - a.pairs;
  const T *src = reinterpret_cast<const T *>(a.qkv) + (long long)tok * a.qkv_stride;
  for (int i = (a.q_out ? 0 : a.n_heads * units) + threadIdx.x; i < heads * units; i += blockDim.x) {
    const int h = i / units, u = i - h * units;
    const bool pair = u < a.pairs, key = h < a.n_heads + Hkv;
    const int first = pair ? u : u + a.pairs, second = first + a.pairs;
    const T *s = src + h * D;
    T x = s[first], y = pair ? s[second] : x;
    if (pair && key) {
      const float2 c = cs[u];
      const float p = to_f32(x), q = to_f32(y);
      x = from_f32<T>(p * c.x - q * c.y);
      y = from_f32<T>(q * c.x + p * c.y);
    }
    T *d;
    if (h < a.n_heads) {
      d = reinterpret_cast<T *>(a.q_out) + (long long)tok * a.q_stride + h * D;
    } else {
      if (page < 0) continue;
      d = reinterpret_cast<T *>((key ? a.pg.k : a.pg.v) + slot_offset(a.pg, page, h - a.n_heads - (key ? 0 : Hkv), (int)slot));
    }
    d[first] = x;
    if (pair) d[second] = y;
  }
}

template <typename T>
static void launch_rope_append(cudaStream_t s, RopeAppendArgs &a, int D) {
  constexpr int V = Pack16<T>::N;
  if (a.half && a.pairs % V) {
    rope_append_odd_kernel<T><<<a.tokens, 256, 0, s>>>(a, D);
    return;
  }
  const int units = a.half ? (D - a.pairs) / V : D / V, heads = a.n_heads + 2 * a.pg.n_kv_heads;
  const int rounds = (heads + 256 / units - 1) / (256 / units);      // of a thread over the heads; the same number for each
  a.head_lanes = (heads + rounds - 1) / rounds;
  a.token_lanes = 256 / (units * a.head_lanes);
  if (a.token_lanes > a.tokens) a.token_lanes = a.tokens;
  const int threads = (units * a.head_lanes * a.token_lanes + 31) / 32 * 32;
  const unsigned grid = (unsigned)((a.tokens + a.token_lanes - 1) / a.token_lanes);
  const size_t smem = sizeof(float2) * a.token_lanes * a.pairs;
  if (a.half) rope_append_kernel<T, true><<<grid, threads, smem, s>>>(a, D);
  else rope_append_kernel<T, false><<<grid, threads, smem, s>>>(a, D);
}

}  // namespace tsfm
