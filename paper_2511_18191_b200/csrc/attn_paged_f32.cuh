// The fp32 kernel of tsfm_paged_attention (work split and join: attn_paged.cuh, tiles: attn_paged_fetch.cuh): FMA.
//
// WR x WK warps: a warp takes up to 4 query rows against 64 / WK of a tile's slots.  Eight lanes share a slot, a warp works on 8 or 16 at a
// time, two or four a group of eight lanes, each group with its own running maximum and sum; groups, then warps, are merged when the unit ends.
// Bound: memory up to 4 rows (64 x 8 heads of 2048 slots of 64: 88 us, 6.1 TB/s; 32 x 8 heads of 4096 slots of 128, 4 rows: 180 us, 6.0 TB/s;
// loads straight into registers 151 and 252; by cp.async, pages of 4 slots, 249 against 203 after a flush of L2).  Above: instructions and their
// chains, not FMAs (64 x 20 heads of 329 slots of 64, 9 rows: 187 us, of which the products are some 25 at the 16 rows that they are padded to):
// eight lanes repeat each row's maximum and exponentials, and a score takes three shuffles in a row.  Scores kept for the weights: 929 us for 32
// series of up to 16001 slots, 4 heads of 64, 20 rows.
#pragma once
#include "attn_paged_fetch.cuh"

namespace tsfm {

template <int D_, int WROWS_, int WR_> struct PagedF32 {
  static constexpr int D = D_, WROWS = WROWS_, WR = WR_;
  static constexpr int WARPS = D == 128 ? 8 : 4, WK = WARPS / WR, THREADS = 32 * WARPS + 32, KEYS = PA_TILE / WK;
  static constexpr int ROWS = WROWS * WR, RB = D * 4;
  static constexpr int N = WROWS == 1 && KEYS >= 16 ? 4 : 2;       // slots of a group at once
  static_assert(KEYS % (4 * N) == 0, "a warp stays within its slots");
  static constexpr bool Q_SHARED = D == 128 && WROWS == 4;        // four rows of queries beside four of sums would not fit the registers
  static constexpr int PD = 32, PARTS = D / PD, PB = PD * 4, PART_BYTES = PA_TILE * PB;
  static constexpr int KV_BYTES = PA_TILE * RB, Q_BYTES = ROWS * RB;
  static constexpr int STAGE_BYTES = (2 * KV_BYTES + Q_BYTES + 1023) / 1024 * 1024;
  static_assert(WARPS * WROWS * (D * 4 + 8) <= STAGE_BYTES, "the merge takes one stage");
  static constexpr int STAGES = D == 128 && WR == 4 ? 2 : 3;
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + (Q_SHARED ? WARPS * WROWS * RB : 0) + 1024;      // (stages begin at multiples of 1 KB)
  static_assert(SMEM_BYTES + 2048 <= 227 * 1024, "a CTA's shared memory");
  static constexpr int CTAS = D == 128 ? 1 : D == 64 ? 2 : 4;
};

template <typename C, bool TMA>
__global__ void __launch_bounds__(C::THREADS, C::CTAS) paged_attn_f32_kernel(const __grid_constant__ PagedAttnArgs a, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV) {
  constexpr int D = C::D, S = C::STAGES, WK = C::WK, WARPS = C::WARPS, WROWS = C::WROWS, ROWS = C::ROWS, PARTS = C::PARTS, PB = C::PB;
  constexpr int E = D / 8, N = C::N;               // elements of a lane; slots of a group at once
  constexpr int FULL = bar_full(), EMPTY = bar_empty(S), MERGE = bar_merge(S);
  extern __shared__ __align__(1024) unsigned char paged_smem_raw[];
  __shared__ PagedStages<S, TMA> sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wr = warp / WK, wk = warp % WK, l8 = lane & 7, grp = lane >> 3;
  const uint32_t smem0 = (smem_u32(paged_smem_raw) + 1023u) & ~1023u;
  unsigned char *const smem = paged_smem_raw + (smem0 - smem_u32(paged_smem_raw));
  const int R = a.M * a.group;
  const PagedRun run = paged_find_run<C::THREADS>(a);
  pdl_release();                                   // (the join waits for this grid's end; its CTAs may take their places)
  if (tid == 0) {
    PagedMeta meta{-1, 0, 0, 0};
    if (run.count > 0 && run.first) {
      const int tiles = paged_span(a, run.b, false).tiles;
      meta = PagedMeta{run.b, run.u, (int)(run.unit0 / run.per), (int)min((run.unit0 + tiles - 1) / run.per, (long long)gridDim.x - 1)};
    }
    a.meta[blockIdx.x] = meta;
  }
  if (run.count == 0) return;
  if (warp == WARPS) {
    paged_fetch<C, TMA>(a, run, sh, smem0, mapK, mapV);
    return;
  }

  float q[C::Q_SHARED ? 1 : WROWS][E], o[WROWS][E], m[WROWS], l[WROWS];
  float4 *const q_own = reinterpret_cast<float4 *>(smem + S * C::STAGE_BYTES + warp * WROWS * C::RB) + l8;        // [row][part][8]
  int2 range[WROWS];
  int min_end = 0, max_start = 0, total = 0, tile0 = 0, tiles = 0, seg_first = 0, n_new = 0, h = 0, row0 = 0, stage = 0;
#pragma unroll 1
  for (int i = 0; i < run.count; ++i) {
    bar_sync(FULL + stage, C::THREADS);
    const PagedItem it = sh.item[stage];
    unsigned char *const keys = smem + stage * C::STAGE_BYTES;
    if (it.first) {
      const PagedSpan s = it.sp;
      h = it.u / a.chunks, row0 = (it.u - h * a.chunks) * ROWS;
      total = s.total, tile0 = s.tile0, tiles = s.tiles, n_new = s.n_new, seg_first = it.t;
      min_end = paged_row_range(a, s, token_of(a, row0)).y;
      max_start = paged_row_range(a, s, min(s.n_new, token_of(a, min(R, row0 + ROWS) - 1) + 1) - 1).x;
#pragma unroll
      for (int r = 0; r < WROWS; ++r) {
        const int own = wr * WROWS + r, row = row0 + own;
        range[r] = row < R ? paged_row_range(a, s, token_of(a, row)) : make_int2(0, 0);
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          const float4 x = *reinterpret_cast<const float4 *>(keys + 2 * C::KV_BYTES + own * C::RB + query_swz<C::RB>(own, p * 8 + l8) * 16);
          if (C::Q_SHARED) q_own[(r * PARTS + p) * 8] = x;     // (all groups of a warp the same value)
          else q[C::Q_SHARED ? 0 : r][4 * p] = x.x, q[C::Q_SHARED ? 0 : r][4 * p + 1] = x.y, q[C::Q_SHARED ? 0 : r][4 * p + 2] = x.z, q[C::Q_SHARED ? 0 : r][4 * p + 3] = x.w;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) o[r][e] = 0.f;
      }
    }
    const int base = (tile0 + it.t) * PA_TILE;
    const unsigned long long valid = sh.valid[stage][0] | (unsigned long long)sh.valid[stage][1] << 32;
    const bool open = valid == ~0ull && base >= max_start && base + PA_TILE <= min_end;      // every row sees every slot
#pragma unroll 1
    for (int k0 = wk * C::KEYS; k0 < (wk + 1) * C::KEYS; k0 += 4 * N) {
      float sc[N][WROWS];
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int r = 0; r < WROWS; ++r) sc[j][r] = 0.f;
#pragma unroll(C::Q_SHARED ? 1 : PARTS)
      for (int p = 0; p < PARTS; ++p) {
        float4 x[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const int at = k0 + 4 * j + grp;
          x[j] = *reinterpret_cast<const float4 *>(keys + p * C::PART_BYTES + at * PB + tile_swz<PB>(at, l8) * 16);
        }
#pragma unroll
        for (int r = 0; r < WROWS; ++r) {
          float4 y;
          if (C::Q_SHARED) y = q_own[(r * PARTS + p) * 8];
          else y = make_float4(q[C::Q_SHARED ? 0 : r][4 * p], q[C::Q_SHARED ? 0 : r][4 * p + 1], q[C::Q_SHARED ? 0 : r][4 * p + 2], q[C::Q_SHARED ? 0 : r][4 * p + 3]);
#pragma unroll
          for (int j = 0; j < N; ++j) sc[j][r] = fmaf(y.x, x[j].x, fmaf(y.y, x[j].y, fmaf(y.z, x[j].z, fmaf(y.w, x[j].w, sc[j][r]))));
        }
      }
#pragma unroll
      for (int x = 1; x < 8; x <<= 1)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int r = 0; r < WROWS; ++r) sc[j][r] += __shfl_xor_sync(0xffffffffu, sc[j][r], x);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int at = k0 + 4 * j + grp, slot = base + at;
#pragma unroll
        for (int r = 0; r < WROWS; ++r) {
          sc[j][r] *= a.scale2;
          if (!open && (slot < range[r].x || slot >= range[r].y || !(valid >> at & 1))) sc[j][r] = -INFINITY;
        }
        if (a.scores && l8 == 0 && slot < total) {
#pragma unroll
          for (int r = 0; r < WROWS; ++r) {
            const int row = row0 + wr * WROWS + r;
            if (row < R) a.scores[(((long long)it.b * a.pg.n_kv_heads + h) * R + row) * a.score_stride + slot] = sc[j][r];
          }
        }
      }
      bool moved = false;
      float corr[WROWS];
#pragma unroll
      for (int r = 0; r < WROWS; ++r) {
        float top = m[r];
#pragma unroll
        for (int j = 0; j < N; ++j) top = fmaxf(top, sc[j][r]);
        const float ref = top == -INFINITY ? 0.f : top;
        corr[r] = exp2f(m[r] - ref);
        moved |= corr[r] != 1.f;
        m[r] = top;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) sum += sc[j][r] = exp2f(sc[j][r] - ref);
        l[r] = fmaf(l[r], corr[r], sum);
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int r = 0; r < WROWS; ++r)
#pragma unroll
          for (int e = 0; e < E; ++e) o[r][e] *= corr[r];
      }
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int at = k0 + 4 * j + grp, slot = base + at;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          const float4 x = *reinterpret_cast<const float4 *>(keys + C::KV_BYTES + p * C::PART_BYTES + at * PB + tile_swz<PB>(at, l8) * 16);
#pragma unroll
          for (int r = 0; r < WROWS; ++r) {
            // (a slot that this row does not see may hold anything: 0 x NaN must not happen)
            if (!open && (slot < range[r].x || slot >= range[r].y || !(valid >> at & 1))) continue;
            o[r][4 * p] = fmaf(sc[j][r], x.x, o[r][4 * p]), o[r][4 * p + 1] = fmaf(sc[j][r], x.y, o[r][4 * p + 1]);
            o[r][4 * p + 2] = fmaf(sc[j][r], x.z, o[r][4 * p + 2]), o[r][4 * p + 3] = fmaf(sc[j][r], x.w, o[r][4 * p + 3]);
          }
        }
      }
    }

    if (it.t + 1 == tiles || i + 1 == run.count) {
      // the unit, or this CTA's part of it, ends: the four groups of a warp, then the warps through this stage's memory
      const int rows = min(ROWS, R - row0);
      bar_sync(MERGE, 32 * WARPS);
      float *scratch = reinterpret_cast<float *>(keys);                      // [warp][row][D]
      float2 *ml_scratch = reinterpret_cast<float2 *>(scratch + WARPS * WROWS * D);
#pragma unroll
      for (int r = 0; r < WROWS; ++r) {
        if (TMA && sh.dead) l[r] = NAN;
#pragma unroll
        for (int x = 8; x < 32; x <<= 1) {
          const float om = __shfl_xor_sync(0xffffffffu, m[r], x), ol = __shfl_xor_sync(0xffffffffu, l[r], x);
          const float top = fmaxf(m[r], om), ref = top == -INFINITY ? 0.f : top;
          const float f0 = exp2f(m[r] - ref), f1 = exp2f(om - ref);
          m[r] = top;
          l[r] = l[r] * f0 + ol * f1;
#pragma unroll
          for (int e = 0; e < E; ++e) o[r][e] = o[r][e] * f0 + __shfl_xor_sync(0xffffffffu, o[r][e], x) * f1;
        }
        if (grp == 0) {
#pragma unroll
          for (int p = 0; p < PARTS; ++p)
            *reinterpret_cast<float4 *>(scratch + (warp * WROWS + r) * D + p * 32 + l8 * 4) = make_float4(o[r][4 * p], o[r][4 * p + 1], o[r][4 * p + 2], o[r][4 * p + 3]);
          if (l8 == 0) ml_scratch[warp * WROWS + r] = make_float2(m[r], l[r]);
        }
      }
      bar_sync(MERGE, 32 * WARPS);
      const bool whole = seg_first == 0 && it.t + 1 == tiles;
      const int part = 2 * blockIdx.x + (seg_first == 0);
      for (int e = tid; e < rows * (D / 4); e += 32 * WARPS) {
        const int r = e / (D / 4), d = e % (D / 4) * 4, w0 = r / WROWS * WK, rl = r % WROWS;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < WK; ++w) top = fmaxf(top, ml_scratch[(w0 + w) * WROWS + rl].x);
        const float ref = top == -INFINITY ? 0.f : top;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WK; ++w) {
          const float2 ml = ml_scratch[(w0 + w) * WROWS + rl];
          const float f = exp2f(ml.x - ref);
          const float4 x = *reinterpret_cast<const float4 *>(scratch + ((w0 + w) * WROWS + rl) * D + d);
          sum = fmaf(ml.y, f, sum);
          v.x = fmaf(x.x, f, v.x), v.y = fmaf(x.y, f, v.y), v.z = fmaf(x.z, f, v.z), v.w = fmaf(x.w, f, v.w);
        }
        if (!whole) {
          *reinterpret_cast<float4 *>(a.part_o + ((long long)part * ROWS + r) * D + d) = v;
          if (d == 0) a.part_ml[part * ROWS + r] = make_float2(top, sum);
        } else if (token_of(a, row0 + r) < n_new) {
          const float4 y = sum == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v.x / sum, v.y / sum, v.z / sum, v.w / sum);
          *reinterpret_cast<float4 *>(paged_out_row<float>(a, it.b, h, row0 + r, D) + d) = y;
          if (d == 0) paged_write_lse(a, it.b, h, row0 + r, top, sum);
        }
      }
    }
    if (i + S < run.count) {
      if (TMA) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");        // sums that were written here, before the next tile
      bar_arrive(EMPTY + stage, C::THREADS);
    }
    if (++stage == S) stage = 0;
  }
}

}  // namespace tsfm
