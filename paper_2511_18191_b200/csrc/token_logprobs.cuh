// Log probabilities of given tokens, entropy and the best tokens of rows of logits (tsfm_token_logprobs).
#pragma once
#include <cooperative_groups.h>
#include "pages.cuh"

namespace tsfm {

struct LogprobArgs {
  const void *x;
  long long stride;                                // elements
  int V;
  float scale, scale2;                             // scale2 = scale * log2(e): exponents are kept in base 2
  const int *tokens;
  int n_tokens;
  float *logprob, *lse, *entropy;                  // each or NULL
  int n_top, *ids;
  float *best;
};

constexpr int LP_THREADS = 256, LP_WARPS = LP_THREADS / 32, LP_MAX_CLUSTER = 8, LP_MAX_TOP = 32, LP_ROOM = 512;

// 16 entries of a thread at a time, the next 16 on their way; CTAs on an SM.
template <typename T> struct LogprobShape {
  static constexpr int U = (int)sizeof(T), CTAS = sizeof(T) == 2 ? 5 : 4;        // vectors at a time
};

// One number for an entry: the larger the logit the larger, among equals the lower the token the larger; never 0.  -0 equals 0, NaN lies below
// -inf.
__device__ __forceinline__ unsigned long long logit_key(float x, int id) {
  const uint32_t u = __float_as_uint(x + 0.f);
  const uint32_t rank = isnan(x) ? 0u : u & 0x80000000u ? ~u : u | 0x80000000u;
  return (unsigned long long)rank << 32 | (uint32_t)~id;
}
__device__ __forceinline__ int key_id(unsigned long long key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float key_logit(unsigned long long key) {
  const uint32_t r = (uint32_t)(key >> 32);
  return __uint_as_float(r & 0x80000000u ? r & 0x7fffffffu : ~r);        // (rank 0 gives a NaN)
}

__device__ __forceinline__ float max_or_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// (x - m) scale.  Halves are subtracted: logits of the type's largest and lowest value are further apart than the largest float.
__device__ __forceinline__ float logit_gap(float x, float m, float scale) { return 2.f * ((0.5f * x - 0.5f * m) * scale); }

// Reference logit m, sum of 2^d and sum of d 2^d over d = (logit - m) scale2.  (The difference comes first: logits of the type's lowest value times
// scale2 would be -inf, and a row of nothing else is an even distribution.)
struct LogSum {
  float m, s, t;
};
__device__ __forceinline__ LogSum log_sum_join(const LogSum &a, const LogSum &b, float scale2) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return LogSum{m, a.s + b.s, a.t + b.t};            // (zeros, or NaN)
  LogSum r{m, 0.f, 0.f};
  auto add = [&](const LogSum &x) {
    const float d = x.m == -INFINITY ? 0.f : max_or_nan(logit_gap(x.m, m, scale2), -300.f), f = x.m == -INFINITY ? 1.f : exp2f(d);
    r.s = fmaf(x.s, f, r.s);
    r.t += f * fmaf(x.s, d, x.t);
  };
  add(a);
  add(b);
  return r;
}

__device__ __forceinline__ float lp_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Elements 2 i and 2 i + 1 of a vector, the largest of a vector (NaN aside).
__device__ __forceinline__ float2 logits_of(const uint4 &v, int i, bf16) {
  const uint32_t w = (&v.x)[i];
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 logits_of(const uint4 &v, int i, float) {
  return make_float2(__uint_as_float((&v.x)[2 * i]), __uint_as_float((&v.x)[2 * i + 1]));
}
template <int U> __device__ __forceinline__ float largest(const uint4 (&v)[U], bf16) {
  __nv_bfloat162 m = *reinterpret_cast<const __nv_bfloat162 *>(&v[0].x);
#pragma unroll
  for (int j = 0; j < U; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __hmax2(m, *reinterpret_cast<const __nv_bfloat162 *>(&(&v[j].x)[i]));
  return fmaxf(__low2float(m), __high2float(m));
}
template <int U> __device__ __forceinline__ float largest(const uint4 (&v)[U], float) {
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < U; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(m, __uint_as_float((&v[j].x)[i]));
  return m;
}

// Two elements as floats, -inf as something finite (NaN stays).
constexpr float LP_FAR = 1e30f;
__device__ __forceinline__ float2 finite_logits(const uint4 &v, int i, bf16) {
  const __nv_bfloat162 far = __float2bfloat162_rn(-LP_FAR);
  const __nv_bfloat162 y = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162 *>(&(&v.x)[i]), far);
  const uint32_t w = *reinterpret_cast<const uint32_t *>(&y);
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 finite_logits(const uint4 &v, int i, float) {
  return make_float2(max_or_nan(__uint_as_float((&v.x)[2 * i]), -LP_FAR), max_or_nan(__uint_as_float((&v.x)[2 * i + 1]), -LP_FAR));
}

// Descending order of a warp's keys that rise and then fall, or the other way round.
__device__ __forceinline__ unsigned long long warp_merge(unsigned long long key, int lane) {
#pragma unroll
  for (int j = 16; j; j >>= 1) {
    const unsigned long long other = __shfl_xor_sync(0xffffffffu, key, j);
    if ((key < other) == !(lane & j)) key = other;
  }
  return key;
}
// Descending order of a warp's keys.
__device__ __forceinline__ unsigned long long warp_sort(unsigned long long key, int lane) {
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j; j >>= 1) {
      const unsigned long long other = __shfl_xor_sync(0xffffffffu, key, j);
      const bool up = (lane & k) != 0 && k < 32, first = !(lane & j);    // runs alternate until the last merge
      if ((key < other) == (first != up)) key = other;
    }
  return key;
}

// A cluster of CTAs a row.  One pass over the logits: a thread keeps a reference (its maximum as it was when that last moved), the sum of
// exponentials, the sum of d times them for the entropy, and which of its batches held its largest logit: nothing is done for the best tokens
// while the row streams.  Behind it every thread's largest entry is one key; the n best keys' threads hold all of the n best entries (any
// other entry lies below n of those keys), and only their columns are looked at again, from L2.
// Bound: instructions (of a lane, executed an entry: bf16 12.2 without best tokens and 13.8 with ten, 0.73 to 0.79 issued a cycle; fp32 14.0 and 15.6; the
// exponentials alone, 16 a cycle, take 45 us).  2048 rows of 100003 in bf16: 92 us without best tokens, 112 with 10 of them, 3.7 TB/s; 1024 rows of 100000 in fp32 75 and
// 99.  Two vectors of bf16 a thread ahead and five CTAs on an SM: four and four took 121,
// rows taken in turn by resident CTAs 117 to 130.
template <typename T>
__global__ void __launch_bounds__(LP_THREADS, LogprobShape<T>::CTAS) token_logprobs_kernel(const __grid_constant__ LogprobArgs a) {
  namespace cg = cooperative_groups;
  constexpr int N = 16 / (int)sizeof(T), U = LogprobShape<T>::U, STEP = LP_THREADS * U;
  __shared__ LogSum part[LP_WARPS], whole;
  __shared__ unsigned long long keys[LP_WARPS * LP_MAX_TOP], found[LP_ROOM], top[LP_MAX_TOP];
  __shared__ int columns[LP_MAX_TOP], n_found;
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), c = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = a.V, n = a.n_top;
  const long long row = blockIdx.x / C;
  const T *x = reinterpret_cast<const T *>(a.x) + row * a.stride;
  // vectors at multiples of 16 bytes; vector v holds entries v N - shift ..
  const int shift = (int)((uintptr_t)x & 15) / (int)sizeof(T), vectors = (V + shift + N - 1) / N, slice = (vectors + C - 1) / C;
  const int v0 = min(vectors, c * slice), v1 = min(vectors, v0 + slice);
  auto load = [&](int v) {                         // entries that do not exist are -inf
    uint4 r;
    const int first = v * N - shift;
    if (v < v1 && first >= 0 && first + N <= V) {
      r = __ldg(reinterpret_cast<const uint4 *>(x + first));
    } else {
      T *e = reinterpret_cast<T *>(&r);
#pragma unroll
      for (int i = 0; i < N; ++i) e[i] = v < v1 && first + i >= 0 && first + i < V ? x[first + i] : from_f32<T>(-INFINITY);
    }
    return r;
  };
  float m = -INFINITY;                             // the largest logit so far above -1e30
  int from = -1;                                   // the batch that holds it
  LogSum mine;
  bool extreme = a.scale2 >= 1e6f;                 // a maximum, or a scale, with which y scale2 - m scale2 could overflow or -1e30 be more than nothing
  {
    float ref = 0.f;                               // m scale2 as rounded
    float ss[2] = {0.f, 0.f}, tt[2] = {0.f, 0.f};
    uint4 r[U], next[U];
#pragma unroll
    for (int j = 0; j < U; ++j) next[j] = load(v0 + tid + j * LP_THREADS);
    for (int v = v0 + tid; v < v1; v += STEP) {
#pragma unroll
      for (int j = 0; j < U; ++j) r[j] = next[j];
      if (v + STEP < v1) {
#pragma unroll
        for (int j = 0; j < U; ++j) next[j] = load(v + STEP + j * LP_THREADS);
      }
      const float big = largest(r, T());
      if (big > m && big > -LP_FAR) {
        const float now = big * a.scale2, d = ref - now, f = m == -INFINITY ? 0.f : lp_ex2(d);
        // (before the first number the sums are 0, or NaN)
        const float s = ss[0] + ss[1], t = tt[0] + tt[1];
        ss[0] = m == -INFINITY ? s : s * f, tt[0] = m == -INFINITY ? t : f == 0.f ? 0.f * t : f * fmaf(s, d, t);
        ss[1] = tt[1] = 0.f;
        m = big, ref = now, from = v;
        // (from 2^31 on what rounding left of ref, up to 64, could overflow as an exponent)
        extreme |= big >= LP_FAR || fabsf(now) >= 2147483648.f;
      }
      float bs[2] = {0.f, 0.f}, bt[2] = {0.f, 0.f};        // (of the batch: shorter sums lose less)
#pragma unroll
      for (int j = 0; j < U; ++j)
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          const float2 y = finite_logits(r[j], i, T());
          const float d0 = fmaf(y.x, a.scale2, -ref), d1 = fmaf(y.y, a.scale2, -ref);
          const float e0 = lp_ex2(d0), e1 = lp_ex2(d1);
          bs[0] += e0, bs[1] += e1;
          bt[0] = fmaf(e0, d0, bt[0]), bt[1] = fmaf(e1, d1, bt[1]);
        }
      ss[0] += bs[0], ss[1] += bs[1], tt[0] += bt[0], tt[1] += bt[1];
    }
    // against m itself, not against its rounded product
    const float s = ss[0] + ss[1], t = tt[0] + tt[1];
    const float off = m == -INFINITY ? 0.f : fmaf(m, a.scale2, -ref), f = exp2f(-off);
    // what stands for -inf has to count as nothing beside m, or beside 0 before there is one
    extreme |= ((m == -INFINITY ? 0.f : m) + LP_FAR) * a.scale2 < 300.f;
    mine = LogSum{m, s * f, fmaf(-off, s, t) * f};
  }
  const bool far = __syncthreads_or(extreme) || !__syncthreads_or(from >= 0);
  if (far) {                                       // logits beyond 1e30, or none above -1e30: once more, the difference first
    uint64_t s2 = 0, t2 = 0;
    m = -INFINITY;
    for (int v = v0 + tid; v < v1; v += LP_THREADS) {
      const uint4 r[1] = {load(v)};
      m = fmaxf(m, largest(r, T()));
    }
    from = -1;
    const float ref = m == -INFINITY ? 0.f : -0.5f * m;
    for (int v = v0 + tid; v < v1; v += LP_THREADS) {
      const uint4 r = load(v);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const float2 y = logits_of(r, i, T());
        float2 d = unpack2(mul2(fma2(f32x2(y.x, y.y), f32x2(0.5f, 0.5f), f32x2(ref, ref)), f32x2(a.scale2, a.scale2)));
        d.x += d.x, d.y += d.y;                    // (halves: as logit_gap)
        d.x = max_or_nan(d.x, -300.f), d.y = max_or_nan(d.y, -300.f);    // (2^-300 is 0, and -inf times it must be too)
        const uint64_t e = f32x2(lp_ex2(d.x), lp_ex2(d.y));
        s2 = add2(s2, e);
        t2 = fma2(e, f32x2(d.x, d.y), t2);
      }
    }
    const float2 s = unpack2(s2), t = unpack2(t2);
    mine = LogSum{m, s.x + s.y, t.x + t.y};
  }
  {
#pragma unroll
    for (int o = 16; o; o >>= 1)
      mine = log_sum_join(mine, LogSum{__shfl_xor_sync(0xffffffffu, mine.m, o), __shfl_xor_sync(0xffffffffu, mine.s, o), __shfl_xor_sync(0xffffffffu, mine.t, o)}, a.scale2);
    if (lane == 0) part[warp] = mine;
  }
  unsigned long long best = 0;
  if (n) {
    // this thread's best entry
    unsigned long long key = 0;
    if (from >= 0) {
      int id = 0;
#pragma unroll
      for (int j = U - 1; j >= 0; --j) {
        const uint4 r = load(from + j * LP_THREADS);
#pragma unroll
        for (int i = N / 2 - 1; i >= 0; --i) {
          const float2 y = logits_of(r, i, T());
          const int at = (from + j * LP_THREADS) * N - shift + 2 * i;
          id = y.x == m ? at : y.y == m ? at + 1 : id;
        }
      }
      key = logit_key(m, id);
    } else {                                       // (nothing above -inf: all of them)
      for (int v = v0 + tid; v < v1; v += LP_THREADS) {
        const uint4 r = load(v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int id = v * N - shift + i;
          if (id >= 0 && id < V) key = max(key, logit_key(to_f32(reinterpret_cast<const T *>(&r)[i]), id));
        }
      }
    }
    key = warp_sort(key, lane);
    best = key;
    keys[warp * 32 + lane] = key;
    if (tid < LP_MAX_TOP) columns[tid] = -1, top[tid] = 0;
    if (tid == 0) n_found = 0;
  }
  __syncthreads();
  if (warp == 0) {
    LogSum all = lane < LP_WARPS ? part[lane] : LogSum{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int o = 16; o; o >>= 1)
      all = log_sum_join(all, LogSum{__shfl_xor_sync(0xffffffffu, all.m, o), __shfl_xor_sync(0xffffffffu, all.s, o), __shfl_xor_sync(0xffffffffu, all.t, o)}, a.scale2);
    if (lane == 0) whole = all;
  }
  if (n) {
    auto place = [&](const unsigned long long *list, int count, unsigned long long key) {        // how many of the list are larger
      int above = 0;
      for (int i = 0; i < count; ++i) above += list[i] > key;
      return above;
    };
    // the warps' lists become one: the larger of one from the top and the other from the bottom are the best 32, rising and falling
    __shared__ unsigned long long least;
#pragma unroll
    for (int w = LP_WARPS / 2; w; w >>= 1) {
      if (warp < w) keys[warp * 32 + lane] = best = warp_merge(max(best, keys[(warp + w) * 32 + 31 - lane]), lane);
      __syncthreads();
    }
    if (warp == 0 && lane < n) {
      if (best) columns[lane] = ((key_id(best) + shift) / N - v0) % LP_THREADS;
      if (lane == n - 1) least = best;
    }
    __syncthreads();
    const unsigned long long bar = max(least, 1ull);                     // (fewer keys than n: everything counts)
    const float low = key_logit(bar);                                    // (NaN: below everything)
    for (int k = warp; k < n && columns[k] >= 0; k += LP_WARPS)
      for (int v = v0 + columns[k] + lane * LP_THREADS; v < v1; v += 32 * LP_THREADS) {
        const uint4 r = load(v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float y = to_f32(reinterpret_cast<const T *>(&r)[i]);
          if (y < low) continue;
          const int id = v * N - shift + i;
          const unsigned long long key = id >= 0 && id < V ? logit_key(y, id) : 0;
          if (key >= bar) {
            const int at = atomicAdd(&n_found, 1);
            if (at < LP_ROOM) found[at] = key;
          }
        }
      }
    __syncthreads();
    if (n_found <= LP_ROOM) {
      for (int i = tid; i < n_found; i += LP_THREADS) {
        const int at = place(found, n_found, found[i]);
        if (at < n) top[at] = found[i];
      }
    } else {
      // (hundreds of entries above the n-th best key: they crowd in few columns.  One after the other, then.)
      unsigned long long below = ~0ull;
      for (int k = 0; k < n; ++k) {
        unsigned long long key = 0;
        for (int v = v0 + tid; v < v1; v += LP_THREADS) {
          const uint4 r = load(v);
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const int id = v * N - shift + i;
            const unsigned long long e = id >= 0 && id < V ? logit_key(to_f32(reinterpret_cast<const T *>(&r)[i]), id) : 0;
            if (e < below) key = max(key, e);
          }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) key = max(key, __shfl_xor_sync(0xffffffffu, key, o));
        __syncthreads();
        if (lane == 0) keys[warp] = key;
        __syncthreads();
        for (int w = 0; w < LP_WARPS; ++w) key = max(key, keys[w]);
        if (tid == 0) top[k] = key;
        below = key;
      }
    }
  }
  __syncthreads();
  LogSum all = whole;
  if (C > 1) {
    cluster.sync();
    if (c == 0) {
      for (int k = 1; k < C; ++k) all = log_sum_join(all, *cluster.map_shared_rank(&whole, k), a.scale2);
      if (n && tid < C * n) found[tid] = cluster.map_shared_rank(top, tid / n)[tid % n];
    }
    cluster.sync();
    if (c) return;
    if (n) {
      unsigned long long key = tid < C * n ? found[tid] : 0;
      if (tid < n) top[tid] = 0;
      __syncthreads();
      int above = 0;
      for (int i = 0; i < C * n; ++i) above += found[i] > key;
      if (key && above < n) top[above] = key;
      __syncthreads();
    }
  }
  constexpr float LN2 = 0.69314718055994530942f;
  const float log2_s = log2f(all.s);
  // (not in base 2, in which a token at the type's lowest value would be beyond it)
  auto log_prob = [&](float logit) { return all.s == 0.f ? -INFINITY : logit_gap(logit, all.m, a.scale) - log2_s * LN2; };
  if (tid == 0) {
    if (a.lse) a.lse[row] = all.s == 0.f ? -INFINITY : fmaf(all.m, a.scale, log2_s * LN2);
    if (a.entropy) a.entropy[row] = all.s == 0.f ? 0.f : (log2_s - all.t / all.s) * LN2;
  }
  for (int i = tid; i < a.n_tokens; i += LP_THREADS) {
    const int id = a.tokens[row * a.n_tokens + i];
    a.logprob[row * a.n_tokens + i] = (unsigned)id < (unsigned)V ? log_prob(to_f32(x[id])) : -INFINITY;
  }
  if (tid < n) {
    a.ids[row * n + tid] = top[tid] ? key_id(top[tid]) : -1;
    a.best[row * n + tid] = top[tid] ? log_prob(key_logit(top[tid])) : -INFINITY;
  }
}

}  // namespace tsfm
