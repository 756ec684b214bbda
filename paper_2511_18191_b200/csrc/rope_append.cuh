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
  int parts;                                       // warps of a token
  float mscale;
  uint64_t turn[ROPE_MAX_PAIRS];                   // 2^64 x turns a position
};

// cos and sin of position t: the angle in turns is the low 64 bits of t * turn, exact modulo a whole turn, so that far
// positions lose nothing; the upper 32 of them go into the float, which keeps 24 (an angle is off by 2^-25 of half a turn at most).
__device__ __forceinline__ float2 rope_cos_sin(uint64_t turn, long long t, float mscale) {
  const uint64_t phase = turn * (uint64_t)t;
  float s, c;
  sincospif((float)(int)(phase >> 32) * 4.656612873077392578125e-10f, &s, &c);      // 2^-31: half turns
  return make_float2(c * mscale, s * mscale);
}

// Two neighbouring elements as floats, and back.
__device__ __forceinline__ uint64_t pair_in(const Pack16<bf16> &x, int i) {
  const uint32_t w = (&x.raw.x)[i];
  return f32x2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ void pair_out(Pack16<bf16> &x, int i, uint64_t v) {
  const float2 f = unpack2(v);
  const __nv_bfloat162 r = __floats2bfloat162_rn(f.x, f.y);
  (&x.raw.x)[i] = *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint64_t pair_in(const Pack16<float> &x, int i) { return f32x2(x.get(2 * i), x.get(2 * i + 1)); }
__device__ __forceinline__ void pair_out(Pack16<float> &x, int i, uint64_t v) {
  const float2 f = unpack2(v);
  x.set(2 * i, f.x);
  x.set(2 * i + 1, f.y);
}

// A unit is what a lane turns at once in a head: with `half` a vector of the first half and its partner (or a vector behind
// the turned part), interleaved a vector.  A warp takes a token (few tokens: a part of its heads), computes the angles, two a
// lane, and goes over the heads with its lanes' units fixed: a lane holds its angles, the next heads are on their way while
// it turns the last ones, and no warp waits for another.  (With a CTA a token, and its barrier between angles and heads, the
// indices cost as much as the heads: 140 us for 27000 tokens of 48 heads of 128, and a loop over tokens made it 154; so it is 111,
// 5.9 TB/s.)
constexpr int ROPE_WARPS = 8;
template <typename T, bool HALF>
__global__ void __launch_bounds__(32 * ROPE_WARPS) rope_append_kernel(const __grid_constant__ RopeAppendArgs a, int D) {
  constexpr int V = Pack16<T>::N, N = 2;           // elements of a vector; heads of a lane in flight
  constexpr int A = HALF ? V : V / 2;              // angles of a unit
  __shared__ __align__(16) float cs[ROPE_WARPS][2][ROPE_MAX_PAIRS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long task = (long long)blockIdx.x * ROPE_WARPS + warp;
  if (task >= (long long)a.tokens * a.parts) return;
  const int tok = a.parts == 1 ? (int)task : (int)(task / a.parts), part = (int)(task - (long long)tok * a.parts);
  const int b = tok / a.M, m = tok - b * a.M;
  if (a.n_new && m >= a.n_new[b]) return;
  const int vecs = D / V, half_vecs = a.pairs / V;
  const int units = HALF ? vecs - half_vecs : vecs, head_lanes = 32 / units;
  const int hl = lane / units, u = lane - hl * units;
  const int Hkv = a.pg.n_kv_heads, step = a.parts * head_lanes;
  const int heads = hl < head_lanes ? a.n_heads + 2 * Hkv : 0;   // (lanes behind the last whole head have nothing to do)
  const int first = HALF && u >= half_vecs ? u + half_vecs : u;  // this unit's vectors of a head
  const bool pair = HALF && u < half_vecs;
  const int second = first + half_vecs;
  const T *src = reinterpret_cast<const T *>(a.qkv) + (long long)tok * a.qkv_stride;
  Pack16<T> x[N], y[N];
  auto fetch = [&](int h) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const T *s = src + (h + j * step) * D;
      if (h + j * step < heads) {
        x[j].raw = *reinterpret_cast<const uint4 *>(s + first * V);
        if (pair) y[j].raw = *reinterpret_cast<const uint4 *>(s + second * V);
      }
    }
  };
  int h = (a.q_out ? 0 : a.n_heads) + part * head_lanes + hl;
  fetch(h);
  const int length = a.len[b];
  const long long slot = (long long)length + m;
  const bool in = slot >= 0 && slot < a.pg.capacity;
  const int page = in ? page_of(a.pg, a.pg.table + (long long)b * a.pg.table_stride, (int)slot) : -1;
  if (page < 0 && lane == 0) pages_report(a.pg, in ? BAD_ID : BAD_LEN);
  const long long at0 = page < 0 ? 0 : slot_offset(a.pg, page, 0, (int)slot);
  const long long t = (long long)(a.pos ? a.pos[b] : length) + m;
  for (int p = lane; p < a.pairs; p += 32) {
    const float2 c = rope_cos_sin(a.turn[p], t, a.mscale);
    cs[warp][0][p] = c.x;
    cs[warp][1][p] = c.y;
  }
  __syncwarp();
  float c[A], s[A];
  if (pair || !HALF) {
#pragma unroll
    for (int e = 0; e < A; ++e) c[e] = cs[warp][0][min(u * A + e, ROPE_MAX_PAIRS - 1)], s[e] = cs[warp][1][min(u * A + e, ROPE_MAX_PAIRS - 1)];
  }
  T *qdst = a.q_out ? reinterpret_cast<T *>(a.q_out) + (long long)tok * a.q_stride : nullptr;
  for (; h < heads; fetch(h += N * step)) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int hj = h + j * step;
      if (hj >= heads) break;
      if (hj < a.n_heads + Hkv) {
        if (pair) {
#pragma unroll
          for (int e = 0; e < V / 2; ++e) {
            const uint64_t p = pair_in(x[j], e), q = pair_in(y[j], e), cc = f32x2(c[2 * e], c[2 * e + 1]), ss = f32x2(s[2 * e], s[2 * e + 1]);
            pair_out(x[j], e, fma2(p, cc, mul2(q, f32x2(-s[2 * e], -s[2 * e + 1]))));
            pair_out(y[j], e, fma2(q, cc, mul2(p, ss)));
          }
        } else if (!HALF) {
#pragma unroll
          for (int e = 0; e < V / 2; ++e) {
            if (u * A + e < a.pairs) {             // (what does not turn is left alone, NaN included)
              const uint64_t p = pair_in(x[j], e);
              const float2 f = unpack2(p);
              pair_out(x[j], e, fma2(p, f32x2(c[e], c[e]), mul2(f32x2(f.y, f.x), f32x2(-s[e], s[e]))));
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
        d = reinterpret_cast<T *>((key ? a.pg.k : a.pg.v) + at0 + (hj - a.n_heads - (key ? 0 : Hkv)) * a.pg.head_stride);
      }
      *reinterpret_cast<uint4 *>(d + first * V) = x[j].raw;
      if (pair) *reinterpret_cast<uint4 *>(d + second * V) = y[j].raw;
    }
  }
}

// HALF with a half that is no whole number of vectors: element pairs (and the single elements behind the turned part), one
// a thread.  A thread reads both elements of a pair before it writes them, so in place works here too.  Bound: instructions of single
// elements (27000 tokens of 48 heads of 128, 24 of them turned: 421 us after a flush of L2; with 32 turned, by vectors, 144).
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
  // warps of a token: all that its heads can use while those of all tokens do not fill the SMs
  const int rounds = (heads + 32 / units - 1) / (32 / units);
  a.parts = 1;
  while (2 * a.parts <= rounds && (long long)a.tokens * a.parts < 148 * 16) a.parts *= 2;
  const unsigned grid = (unsigned)(((long long)a.tokens * a.parts + ROPE_WARPS - 1) / ROPE_WARPS);
  const int threads = 32 * ROPE_WARPS;
  if (a.half) rope_append_kernel<T, true><<<grid, threads, 0, s>>>(a, D);
  else rope_append_kernel<T, false><<<grid, threads, 0, s>>>(a, D);
}

}  // namespace tsfm
