// The bf16 kernel of tsfm_paged_attention (work split and join: attn_paged.cuh): tiles of 64 slots in shared memory, products on
// mma.sync m16n8k16.
//
// WR x WK warps compute: a warp takes 8 NQ query rows against 64 / WK of a tile's slots, with a running maximum and sum of its own;
// the WK warps of a row are merged when the unit ends.  Slots are the M side of the products and queries the N side (S^T = K Q^T,
// O^T = V^T P^T, P^T by one 8 x 8 transposition per eight slots): rows come in eights, not sixteens, and eight cost half of the
// instructions and registers.  A fifth warp fetches: it looks the pages up, a slot a lane, and brings tiles (and the queries of a
// unit's first one) in by cp.async, up to STAGES - 1 ahead and across unit borders; slots that no row sees arrive as zeros.  Named
// barriers hand the stages over.  Precision: scores of bf16 operands in fp32; probabilities as two bf16 parts, so that only the
// result is rounded.
#pragma once
#include "attn_narrow.cuh"
#include "attn_paged.cuh"

namespace tsfm {

template <int D, int NQ, int WR> struct PagedMma {
  static constexpr int WK = 4 / WR, KEYS = PA_TILE / WK, BLOCKS = KEYS / 16;
  static constexpr int WROWS = 8 * NQ, ROWS = WROWS * WR, RB = D * 2;
  static constexpr int KV_BYTES = PA_TILE * RB, Q_BYTES = ROWS * RB;
  // the merge, through one stage: rows of D + 4 floats (lanes of a store then meet different banks), maximum and sum
  static constexpr int MERGE_ROW = D + 4, MERGE_BYTES = 4 * WROWS * (MERGE_ROW * 4 + 8);
  static constexpr int STAGE_BYTES = ((2 * KV_BYTES + Q_BYTES > MERGE_BYTES ? 2 * KV_BYTES + Q_BYTES : MERGE_BYTES) + 255) / 256 * 256;
  static constexpr int STAGES = D == 128 ? (WR == 1 ? 3 : 2) : D == 64 ? (WR == 1 ? 4 : 3) : 4;
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES;
  // resident CTAs on an SM: beside the stages what describes them, the scan (128 bytes), alignment, and 1 KB that a CTA costs
  static constexpr int BY_SMEM = 228 * 1024 / (SMEM_BYTES + STAGES * 24 + 128 + 256 + 1024);
  static constexpr int CTAS = BY_SMEM < 4 ? BY_SMEM : 4;
};

constexpr int PA_MMA_THREADS = PA_THREADS + 32;

// Barriers between the fetching warp and the others: `full` of a stage, `empty` of a stage; and one among the others.
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// A tile in a stage: unit u of series b, its t-th tile.
struct PagedItem {
  int b, u, t, first;                              // first: its queries come with it
};

template <int D, int NQ, int WR>
__global__ void __launch_bounds__(PA_MMA_THREADS, PagedMma<D, NQ, WR>::CTAS) paged_attn_mma_kernel(const __grid_constant__ PagedAttnArgs a) {
  using C = PagedMma<D, NQ, WR>;
  constexpr int WK = C::WK, KEYS = C::KEYS, NB = C::BLOCKS, ROWS = C::ROWS, WROWS = C::WROWS, RB = C::RB, S = C::STAGES;
  constexpr int FULL = 1, EMPTY = 1 + S, MERGE = 1 + 2 * S;
  extern __shared__ __align__(256) unsigned char paged_smem[];
  __shared__ unsigned s_valid[S][2];               // slots of the tile that exist: in [lo, total), page in the pool
  __shared__ PagedItem s_item[S];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wr = warp / WK, wk = warp % WK;
  const int g = lane >> 2, t4 = lane & 3;
  const uint32_t smem0 = (uint32_t)__cvta_generic_to_shared(paged_smem);
  const int R = a.M * a.group;
  const PagedRun run = paged_find_run<PA_MMA_THREADS>(a);
  if (tid == 0) {
    PagedMeta meta{-1, 0, 0, 0};
    if (run.count > 0 && run.first) {
      const int tiles = paged_span(a, run.b, false).tiles;
      meta = PagedMeta{run.b, run.u, (int)(run.unit0 / run.per), (int)((run.unit0 + tiles - 1) / run.per)};
    }
    a.meta[blockIdx.x] = meta;
  }
  if (run.count == 0) return;

  if (warp == PA_THREADS / 32) {
    constexpr int CPR = D / 8, STEP = 32 / CPR;    // 16-byte chunks of a row; rows of a copy instruction
    const int chunk = lane % CPR, sub = lane / CPR;
    int b = run.b, u = run.u, t = run.first;
    PagedSpan sp = paged_span(a, b, false);
    long long off[2];                              // byte offsets of slots lane, lane + 32 of the next tile; -1: hidden
    auto look_up = [&]() {
      const int *row = a.pg.table + (long long)b * a.pg.table_stride;
      int page[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int slot = (sp.tile0 + t) * PA_TILE + 32 * x + lane;
        page[x] = slot >= sp.lo && slot < sp.total ? page_of(a.pg, row, slot) : -2;
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        off[x] = page[x] < 0 ? -1 : slot_offset(a.pg, page[x], u / a.chunks, (sp.tile0 + t) * PA_TILE + 32 * x + lane);
        if (page[x] == -1) pages_report(a.pg, BAD_ID);
      }
    };
    look_up();
    int stage = 0;
    for (int i = 0; i < run.count; ++i) {
      const uint32_t dst = smem0 + stage * C::STAGE_BYTES;
      if (i >= S) bar_sync(EMPTY + stage, PA_MMA_THREADS);
      const unsigned v0 = __ballot_sync(0xffffffffu, off[0] >= 0), v1 = __ballot_sync(0xffffffffu, off[1] >= 0);
      const bool first = i == 0 || t == 0;
      if (lane == 0) {
        s_valid[stage][0] = v0, s_valid[stage][1] = v1;
        s_item[stage] = PagedItem{b, u, t, first};
      }
#pragma unroll
      for (int r = 0; r < PA_TILE; r += STEP) {
        const long long o = __shfl_sync(0xffffffffu, off[r / 32], (r & 31) + sub);
        const uint32_t at = dst + (r + sub) * RB + flash_swz<D>(r + sub, chunk) * 16;
        const long long from = (o < 0 ? 0 : o) + chunk * 16;
        const int bytes = o < 0 ? 0 : 16;
        asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(at), "l"(a.pg.k + from), "r"(bytes) : "memory");
        asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(at + C::KV_BYTES), "l"(a.pg.v + from), "r"(bytes) : "memory");
      }
      if (first) {
        const int h = u / a.chunks, row0 = (u - h * a.chunks) * ROWS;
#pragma unroll 4
        for (int r = sub; r < ROWS; r += STEP) {
          const bool in = row0 + r < R;
          const int tok = in ? (row0 + r) / a.group : 0, head = h * a.group + (in ? row0 + r - tok * a.group : 0);
          const bf16 *src = reinterpret_cast<const bf16 *>(a.q) + ((long long)b * a.M + tok) * a.q_stride + (long long)head * D + chunk * 8;
          const uint32_t at = dst + 2 * C::KV_BYTES + r * RB + flash_swz<D>(r, chunk) * 16;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(src), "r"(in ? 16 : 0) : "memory");
        }
      }
      flash_commit();
      if (i + 1 < run.count) {
        if (++t == sp.tiles) {
          t = 0;
          if (++u == a.units) {
            u = 0;
            do sp = paged_span(a, ++b, false); while (sp.tiles == 0);        // (there is one: the run goes on)
          }
        }
        look_up();
      }
      if (i >= S - 2) {
        flash_wait<S - 2>();
        __threadfence_block();
        bar_arrive(FULL + (stage + 2) % S, PA_MMA_THREADS);                   // tile i - (S - 2)
      }
      if (++stage == S) stage = 0;
    }
    flash_wait<0>();
    __threadfence_block();
    for (int i = max(0, run.count - (S - 2)); i < run.count; ++i) bar_arrive(FULL + i % S, PA_MMA_THREADS);
    return;
  }

  const FlashLane<D> fl(lane);
  const uint32_t key_at = fl.va, value_at = fl.ka;  // (keys are the M side here: rows and chunks change places)
  uint32_t qf[NQ][D / 16][2];
  float o[NQ][D / 16][4], m[NQ][2], l[NQ][2];      // of queries 2 t4, 2 t4 + 1 of each tile of eight; l of this lane's slots only
  int2 range[NQ][2];                               // what they see
  int min_end = 0, max_start = 0, total = 0, tile0 = 0, tiles = 0, len_lo = 0, seg_first = 0, n_new = 0, h = 0, row0 = 0;
  int stage = 0;
#pragma unroll 1
  for (int i = 0; i < run.count; ++i) {
    bar_sync(FULL + stage, PA_MMA_THREADS);
    const PagedItem it = s_item[stage];
    const uint32_t kst = smem0 + stage * C::STAGE_BYTES, vst = kst + C::KV_BYTES;
    if (it.first) {
      const PagedSpan s = paged_span(a, it.b, false);
      h = it.u / a.chunks, row0 = (it.u - h * a.chunks) * ROWS;
      total = s.total, tile0 = s.tile0, tiles = s.tiles, len_lo = s.lo, n_new = s.n_new, seg_first = it.t;
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int row = row0 + wr * WROWS + q * 8 + t4 * 2 + x;
          range[q][x] = row < R ? paged_row_range(a, s, row / a.group) : make_int2(0, 0);
          m[q][x] = -INFINITY;
          l[q][x] = 0.f;
        }
      min_end = paged_row_range(a, s, row0 / a.group).y;
      max_start = paged_row_range(a, s, min(s.n_new, (min(R, row0 + ROWS) - 1) / a.group + 1) - 1).x;
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const int qrow = wr * WROWS + q * 8 + (lane & 7);
        const uint32_t qa = vst + C::KV_BYTES + qrow * RB + flash_swz<D>(qrow, lane >> 3) * 16;
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) {
          uint32_t b[4];
          flash_ldsm4(qa ^ (uint32_t)(ks * 64), b);
          qf[q][2 * ks][0] = b[0], qf[q][2 * ks][1] = b[1], qf[q][2 * ks + 1][0] = b[2], qf[q][2 * ks + 1][1] = b[3];
        }
#pragma unroll
        for (int n = 0; n < D / 16; ++n) o[q][n][0] = o[q][n][1] = o[q][n][2] = o[q][n][3] = 0.f;
      }
    }
    const int base = (tile0 + it.t) * PA_TILE, mine = base + wk * KEYS;       // slots of the tile, of this warp
    const unsigned long long valid = s_valid[stage][0] | (unsigned long long)s_valid[stage][1] << 32;

    // scores, slots x queries
    float s[NB][NQ][4];
    const uint32_t ka = kst + wk * KEYS * RB + key_at;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) s[n][q][0] = s[n][q][1] = s[n][q][2] = s[n][q][3] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        uint32_t k[4];
        flash_ldsm4((ka + n * 16 * RB) ^ (uint32_t)(ks * 32), k);
#pragma unroll
        for (int q = 0; q < NQ; ++q) mma_bf16_16816(s[n][q], k, qf[q][ks][0], qf[q][ks][1]);
      }
    }
    const bool open = valid == ~0ull && base >= max_start && base + PA_TILE <= min_end;      // every row sees every slot
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[n][q][x] *= a.scale2;
    if (!open) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int at = n * 16 + g + 8 * (x >> 1), slot = mine + at;
            const int2 r = range[q][x & 1];
            if (slot < r.x || slot >= r.y || !(valid >> (wk * KEYS + at) & 1)) s[n][q][x] = -INFINITY;
          }
    }
    if (a.scores) {
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int row = row0 + wr * WROWS + q * 8 + t4 * 2 + x;
          if (row >= R) continue;
          float *dst = a.scores + (((long long)it.b * a.pg.n_kv_heads + h) * R + row) * a.score_stride + mine + g;
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (mine + n * 16 + e * 8 + g < total) dst[n * 16 + e * 8] = s[n][q][2 * e + x];
        }
    }
    // running softmax
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      float alpha[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float top = m[q][x];
#pragma unroll
        for (int n = 0; n < NB; ++n) top = fmaxf(top, fmaxf(s[n][q][x], s[n][q][2 + x]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
        const float ref = top == -INFINITY ? 0.f : top;
        alpha[x] = flash_ex2(m[q][x] - ref);
        m[q][x] = top;
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          s[n][q][x] = flash_ex2(s[n][q][x] - ref);
          s[n][q][2 + x] = flash_ex2(s[n][q][2 + x] - ref);
          sum += s[n][q][x] + s[n][q][2 + x];
        }
        l[q][x] = fmaf(l[q][x], alpha[x], sum);
      }
      if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {       // a new maximum: seldom, after the first tiles
#pragma unroll
        for (int n = 0; n < D / 16; ++n) o[q][n][0] *= alpha[0], o[q][n][1] *= alpha[1], o[q][n][2] *= alpha[0], o[q][n][3] *= alpha[1];
      }
    }

    // Where some rows see a slot and others do not, a value that is not finite must not reach the others as 0 x NaN: such
    // slots (rare) leave the products and are added to the rows that see them.
    unsigned long long odd = 0;
    const int from = max(mine, len_lo), to = min(mine + KEYS, total);
    if (a.M > 1 && (max(from, min_end) < to || from < min(to, max_start))) {
      const unsigned char *rows = paged_smem + (vst - smem0) + wk * KEYS * RB;
      uint32_t hit = 0;
#pragma unroll
      for (int w = 0; w < KEYS * RB / 512; ++w) {
        const uint4 v = *reinterpret_cast<const uint4 *>(rows + (w * 32 + lane) * 16);
        // an exponent of ones, 0x7f80, plus 0x80 reaches the sign bit
        hit |= ((v.x & 0x7f807f80u) + 0x00800080u) | ((v.y & 0x7f807f80u) + 0x00800080u) | ((v.z & 0x7f807f80u) + 0x00800080u) | ((v.w & 0x7f807f80u) + 0x00800080u);
      }
      if (__any_sync(0xffffffffu, hit & 0x80008000u)) {
#pragma unroll 1
        for (int key = 0; key < KEYS; ++key) {
          hit = 0;
          for (int w = lane; w < D / 2; w += 32) hit |= (reinterpret_cast<const uint32_t *>(rows + key * RB)[w] & 0x7f807f80u) + 0x00800080u;
          if (__any_sync(0xffffffffu, hit & 0x80008000u)) odd |= 1ull << key;
        }
      }
    }
    const uint32_t va = vst + wk * KEYS * RB + value_at;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      uint32_t hi[NQ][2], lo[NQ][2];               // slots 2 t4, 2 t4 + 1 (+ 8) x query g, after the transposition
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float p0 = s[n][q][2 * e], p1 = s[n][q][2 * e + 1];
          const uint32_t y = pack_bf16x2(p0, p1);
          hi[q][e] = movmatrix_trans(y);
          lo[q][e] = movmatrix_trans(pack_bf16x2(p0 - __uint_as_float(y << 16), p1 - __uint_as_float(y & 0xffff0000u)));
        }
      uint32_t mask0 = ~0u, mask1 = ~0u;
      if (odd) {
        const unsigned bits = (unsigned)(odd >> (n * 16)) >> (2 * t4);
        mask0 = (bits & 1 ? 0u : 0xffffu) | (bits & 2 ? 0u : 0xffff0000u);
        mask1 = (bits & 256 ? 0u : 0xffffu) | (bits & 512 ? 0u : 0xffff0000u);
      }
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        uint32_t v[4];
        flash_ldsm4_trans((va + n * 16 * RB) ^ (uint32_t)(ks * 32), v);
        if (odd) v[0] &= mask0, v[1] &= mask0, v[2] &= mask1, v[3] &= mask1;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          mma_bf16_16816(o[q][ks], v, hi[q][0], hi[q][1]);
          mma_bf16_16816(o[q][ks], v, lo[q][0], lo[q][1]);
        }
      }
      if (odd) {
#pragma unroll 1
        for (int key = 0; key < 16; ++key) {
          if (!(odd >> (n * 16 + key) & 1)) continue;
          const int slot = mine + n * 16 + key, row = wk * KEYS + n * 16 + key;
          const unsigned char *value = paged_smem + (vst - smem0) + row * RB;
#pragma unroll
          for (int q = 0; q < NQ; ++q)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const float p = __shfl_sync(0xffffffffu, key < 8 ? s[n][q][x] : s[n][q][2 + x], (key & 7) * 4 + t4);
              if (slot < range[q][x].x || slot >= range[q][x].y) continue;
#pragma unroll
              for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  o[q][ks][2 * e + x] = fmaf(p, to_f32(*reinterpret_cast<const bf16 *>(value + flash_swz<D>(row, 2 * ks + e) * 16 + g * 2)), o[q][ks][2 * e + x]);
            }
        }
      }
    }

    if (it.t + 1 == tiles || i + 1 == run.count) {
      // the unit, or this CTA's part of it, ends: all warps' parts through this stage's memory, then the result by all threads
      const int rows = min(ROWS, R - row0);
      bar_sync(MERGE, PA_THREADS);
      float *scratch = reinterpret_cast<float *>(paged_smem + stage * C::STAGE_BYTES);        // [warp][row][D + 4]
      float2 *ml_scratch = reinterpret_cast<float2 *>(scratch + 4 * WROWS * C::MERGE_ROW);    // [warp][row]
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int r = q * 8 + t4 * 2 + x;
          float sum = l[q][x];
          sum += __shfl_xor_sync(0xffffffffu, sum, 4);
          sum += __shfl_xor_sync(0xffffffffu, sum, 8);
          sum += __shfl_xor_sync(0xffffffffu, sum, 16);
          if (wr * WROWS + r < rows) {
            if (g == 0) ml_scratch[warp * WROWS + r] = make_float2(m[q][x], sum);
#pragma unroll
            for (int n = 0; n < D / 16; ++n) {
              scratch[(warp * WROWS + r) * C::MERGE_ROW + n * 16 + g] = o[q][n][x];
              scratch[(warp * WROWS + r) * C::MERGE_ROW + n * 16 + g + 8] = o[q][n][2 + x];
            }
          }
        }
      bar_sync(MERGE, PA_THREADS);
      const bool whole = seg_first == 0 && it.t + 1 == tiles;
      const int part = 2 * blockIdx.x + (seg_first == 0);
      for (int e = tid; e < rows * (D / 4); e += PA_THREADS) {
        const int r = e / (D / 4), d = (e - r * (D / 4)) * 4, w0 = r / WROWS * WK, rl = r % WROWS;
        float top = ml_scratch[w0 * WROWS + rl].x;
#pragma unroll
        for (int w = 1; w < WK; ++w) top = fmaxf(top, ml_scratch[(w0 + w) * WROWS + rl].x);
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WK; ++w) {
          const float2 ml = ml_scratch[(w0 + w) * WROWS + rl];
          const float f = exp2f(ml.x - ref);
          const float4 x = *reinterpret_cast<const float4 *>(scratch + ((w0 + w) * WROWS + rl) * C::MERGE_ROW + d);
          sum = fmaf(ml.y, f, sum);
          v.x = fmaf(x.x, f, v.x), v.y = fmaf(x.y, f, v.y), v.z = fmaf(x.z, f, v.z), v.w = fmaf(x.w, f, v.w);
        }
        if (!whole) {
          *reinterpret_cast<float4 *>(a.part_o + ((long long)part * ROWS + r) * D + d) = v;
          if (d == 0) a.part_ml[part * ROWS + r] = make_float2(top, sum);
        } else if ((row0 + r) / a.group < n_new) {
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          uint2 y = sum == 0.f ? make_uint2(0u, 0u) : make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
          *reinterpret_cast<uint2 *>(paged_out_row<bf16>(a, it.b, h, row0 + r, D) + d) = y;
          if (d == 0) paged_write_lse(a, it.b, h, row0 + r, top, sum);
        }
      }
    }
    if (i + S < run.count) bar_arrive(EMPTY + stage, PA_MMA_THREADS);
    if (++stage == S) stage = 0;
  }
}

}  // namespace tsfm
