// The bf16 kernel of tsfm_paged_attention (work split and join: attn_paged.cuh): tiles of 64 slots in shared memory, products on
// mma.sync m16n8k16.
//
// WR x WK warps compute: a warp takes 8 NQ query rows against 64 / WK of a tile's slots, with a running maximum and sum of its own;
// the WK warps of a row are merged when the unit ends.  Slots are the M side of the products and queries the N side (S^T = K Q^T,
// O^T = V^T P^T, P^T by one 8 x 8 transposition per eight slots): rows come in eights, not sixteens, and eight cost half of the
// instructions and registers.  One more warp fetches (attn_paged_fetch.cuh).  Precision: scores of bf16 operands in fp32;
// probabilities as two bf16 parts, so that only the result is rounded.
// Bound: memory where units are long and rows few (256 series of up to 8192 slots, 8 heads of 128, 4 rows: 465 us, 6.2 TB/s; one series of
// 131071 slots: 83 us, 6.4 TB/s), the chain of a warp with 20 rows (32 series of up to 16001 slots, 4 heads of 64: 95 us, 3.5 TB/s with the
// scores that it writes), and what starts and ends a unit where those are short (9 rows, 4.6 tiles a unit, 20 heads of 64: 32 us, 2.9 TB/s).
// By cp.async, pages of 4 slots, 64 series of up to 8192 slots are as fast as by TMA (138 us against 142).
#pragma once
#include "attn_narrow.cuh"
#include "attn_paged_fetch.cuh"

namespace tsfm {

template <int D_, int NQ_, int WR_, bool TREE_> struct PagedMma {
  static constexpr int D = D_, NQ = NQ_, WR = WR_;
  static constexpr bool TREE = TREE_;              // masks of attn_tree.cuh
  static constexpr int WK = 2, KEYS = PA_TILE / WK, BLOCKS = KEYS / 16;
  static constexpr int WARPS = WR * WK, THREADS = 32 * WARPS + 32;
  static constexpr int WROWS = 8 * NQ, ROWS = WROWS * WR, RB = D * 2;
  static constexpr int PD = D < 64 ? D : 64, PARTS = D / PD, PB = PD * 2, PART_BYTES = PA_TILE * PB;
  static constexpr int KV_BYTES = PA_TILE * RB, Q_BYTES = ROWS * RB;
  // the merge, through one stage: a lane's float4s
  static constexpr int MERGE_WORDS = NQ + NQ * D / 16;
  static constexpr int STAGE_BYTES = (2 * KV_BYTES + Q_BYTES + 1023) / 1024 * 1024;
  static_assert(WR * (WK - 1) * 32 * MERGE_WORDS * 16 <= STAGE_BYTES, "the merge takes one stage");
  static constexpr int STAGES = 3;
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + 1024;        // (stages begin at multiples of 1 KB)
  // resident CTAs on an SM: beside the stages what describes them, the scan (128 bytes), alignment, and 1 KB that a CTA costs
  static constexpr int BY_SMEM = 228 * 1024 / (SMEM_BYTES + STAGES * 128 + 128 + 1024);
  static constexpr int CTAS = D == 128 ? (BY_SMEM < 2 ? BY_SMEM : 2) : BY_SMEM < 4 ? BY_SMEM : 4;
};

template <typename C, bool TMA>
__global__ void __launch_bounds__(C::THREADS, C::CTAS) paged_attn_mma_kernel(const __grid_constant__ PagedAttnArgs a, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV) {
  constexpr int D = C::D, NQ = C::NQ;
  constexpr int WK = C::WK, KEYS = C::KEYS, NB = C::BLOCKS, ROWS = C::ROWS, WROWS = C::WROWS, RB = C::RB, S = C::STAGES;
  constexpr int FULL = bar_full(), EMPTY = bar_empty(S), MERGE = bar_merge(S);
  constexpr int PD = C::PD, PB = C::PB;
  extern __shared__ __align__(1024) unsigned char paged_smem_raw[];
  __shared__ PagedStages<S, TMA> sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wr = warp / WK, wk = warp % WK;
  const int g = lane >> 2, t4 = lane & 3;
  const uint32_t smem0 = (smem_u32(paged_smem_raw) + 1023u) & ~1023u;
  unsigned char *const paged_smem = paged_smem_raw + (smem0 - smem_u32(paged_smem_raw));
  const int R = a.M * a.group;
  PagedRun run;
  if constexpr (C::TREE) run = paged_find_unit_run<C::THREADS>(a, ROWS, 1);
  else run = paged_find_run<C::THREADS>(a);
  pdl_release();                                   // (the join waits for this grid's end; its CTAs may take their places)
  if (tid == 0) {
    PagedMeta meta{-1, 0, 0, 0};
    if (run.count > 0 && run.first) {
      const int tiles = C::TREE ? paged_unit_span(a, run.b, paged_unit_chunk<true>(a, run.u), ROWS, false).tiles : paged_span(a, run.b, false).tiles;
      meta = PagedMeta{run.b, run.u, (int)(run.unit0 / run.per), (int)min((run.unit0 + tiles - 1) / run.per, (long long)gridDim.x - 1)};
    }
    a.meta[blockIdx.x] = meta;
  }
  if (run.count == 0) return;

  if (warp == C::WARPS) {
    paged_fetch<C, TMA>(a, run, sh, smem0, mapK, mapV);
    return;
  }

  const FlashLane<PD> fl(lane);
  const uint32_t key_at = fl.va, value_at = fl.ka;  // (keys are the M side here: rows and chunks change places)
  uint32_t qf[NQ][D / 16][2];
  float o[NQ][D / 16][4], m[NQ][2], l[NQ][2];      // of queries 2 t4, 2 t4 + 1 of each tile of eight; l of this lane's slots only
  int2 range[NQ][2];                               // what they see
  int min_end = 0, max_start = 0, total = 0, tile0 = 0, tiles = 0, len_lo = 0, seg_first = 0, n_new = 0, h = 0, row0 = 0;
  int stage = 0;
#pragma unroll 1
  for (int i = 0; i < run.count; ++i) {
    bar_sync(FULL + stage, C::THREADS);
    const PagedItem it = sh.item[stage];
    const uint32_t kst = smem0 + stage * C::STAGE_BYTES, vst = kst + C::KV_BYTES;
    if (it.first) {
      const PagedSpan s = it.sp;
      h = paged_unit_head<C::TREE>(a, it.u), row0 = paged_unit_chunk<C::TREE>(a, it.u) * ROWS;
      total = s.total, tile0 = s.tile0, tiles = s.tiles, len_lo = s.lo, n_new = s.n_new, seg_first = it.t;
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int row = row0 + wr * WROWS + q * 8 + t4 * 2 + x;
          range[q][x] = row >= R ? make_int2(0, 0) : C::TREE ? paged_tree_range(a, s, it.b, token_of(a, row)) : paged_row_range(a, s, token_of(a, row));
          m[q][x] = -INFINITY;
          l[q][x] = 0.f;
        }
      const int last = min(s.n_new, token_of(a, min(R, row0 + ROWS) - 1) + 1) - 1;
      if constexpr (C::TREE) {
        const int2 open = paged_tree_open(a, s, token_of(a, row0), last);
        max_start = open.x, min_end = open.y;
      } else {
        min_end = paged_row_range(a, s, token_of(a, row0)).y;
        max_start = paged_row_range(a, s, last).x;
      }
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
    const int base = C::TREE ? paged_tile_base<true>(a, it.sp, it.t) : (tile0 + it.t) * PA_TILE, mine = base + wk * KEYS;       // slots of the tile, of this warp
    const unsigned long long valid = sh.valid[stage][0] | (unsigned long long)sh.valid[stage][1] << 32;

    // scores, slots x queries
    float s[NB][NQ][4];
    const uint32_t ka = kst + wk * KEYS * PB + key_at;
    {
      // (two sums each where a warp has few of them: a product waits some 35 cycles for the one before)
      constexpr int CH = NB * NQ < 4 ? 2 : 1;
      float c[CH][NB][NQ][4];
#pragma unroll
      for (int i = 0; i < CH * NB * NQ * 4; ++i) (&c[0][0][0][0])[i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          uint32_t k[4];
          flash_ldsm4((ka + n * 16 * PB + ks / (PD / 16) * C::PART_BYTES) ^ (uint32_t)(ks % (PD / 16) * 32), k);
#pragma unroll
          for (int q = 0; q < NQ; ++q) mma_bf16_16816(c[ks % CH][n][q], k, qf[q][ks][0], qf[q][ks][1]);
        }
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
          for (int x = 0; x < 4; ++x) s[n][q][x] = (CH == 2 ? c[0][n][q][x] + c[CH - 1][n][q][x] : c[0][n][q][x]) * a.scale2;
    }
    const bool open = valid == ~0ull && base >= max_start && base + PA_TILE <= min_end;      // every row sees every slot
    // (of a tree or a window) bits of the warp's slots that row q, x sees
    auto sees = [&](int q, int x) {
      const int row = row0 + wr * WROWS + q * 8 + t4 * 2 + x;
      return (uint32_t)(paged_tree_bits(a, it.sp, range[q][x], it.b, row < R ? token_of(a, row) : a.M, base) >> (wk * KEYS));
    };
    if (!open && C::TREE) {
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint32_t bits = sees(q, x) & (uint32_t)(valid >> (wk * KEYS));
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (!(bits >> (n * 16 + g + 8 * e) & 1)) s[n][q][2 * e + x] = -INFINITY;
        }
    } else if (!open) {
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
    float alpha[NQ][2];
    bool moved = false;
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float top = m[q][x];
#pragma unroll
        for (int n = 0; n < NB; ++n) top = fmaxf(top, fmaxf(s[n][q][x], s[n][q][2 + x]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
        const float ref = top == -INFINITY ? 0.f : top;
        alpha[q][x] = flash_ex2(m[q][x] - ref);
        moved |= alpha[q][x] != 1.f;
        m[q][x] = top;
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          s[n][q][x] = flash_ex2(s[n][q][x] - ref);
          s[n][q][2 + x] = flash_ex2(s[n][q][2 + x] - ref);
          sum += s[n][q][x] + s[n][q][2 + x];
        }
        l[q][x] = fmaf(l[q][x], alpha[q][x], sum);
      }
    if (__any_sync(0xffffffffu, moved)) {          // a new maximum: seldom, after the first tiles
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int n = 0; n < D / 16; ++n) o[q][n][0] *= alpha[q][0], o[q][n][1] *= alpha[q][1], o[q][n][2] *= alpha[q][0], o[q][n][3] *= alpha[q][1];
    }

    // Whole boxes arrive: what lies in slots that no row sees must not reach the products as 0 x NaN.
    unsigned char *const values = paged_smem + (vst - smem0) + wk * KEYS * PB;
    if (TMA && valid != ~0ull) {
      for (int w = lane; w < KEYS * D / 8; w += 32) {
        const int at = w % (KEYS * PD / 8), key = at / (PD / 8);
        if (!(valid >> (wk * KEYS + key) & 1)) *reinterpret_cast<uint4 *>(values + w / (KEYS * PD / 8) * C::PART_BYTES + at * 16) = make_uint4(0u, 0u, 0u, 0u);
      }
      __syncwarp();
    }
    // Where some rows see a slot and others do not, a value that is not finite must not reach the others either: such
    // slots (rare) leave the products and are added to the rows that see them.
    unsigned long long odd = 0;
    const int from = max(mine, len_lo), to = min(mine + KEYS, total);
    // (One token of a chain sees every slot that is valid; one node's mask may hide its own.)
    if (C::TREE ? (a.M > 1 || a.mask) && !open : a.M > 1 && (max(from, min_end) < to || from < min(to, max_start))) {
      uint32_t hit = 0;
#pragma unroll
      for (int w = 0; w < KEYS * D / 256; ++w) {
        const int at = w * 32 + lane;
        const uint4 v = *reinterpret_cast<const uint4 *>(values + at / (KEYS * PD / 8) * C::PART_BYTES + at % (KEYS * PD / 8) * 16);
        // an exponent of ones, 0x7f80, plus 0x80 reaches the sign bit
        hit |= ((v.x & 0x7f807f80u) + 0x00800080u) | ((v.y & 0x7f807f80u) + 0x00800080u) | ((v.z & 0x7f807f80u) + 0x00800080u) | ((v.w & 0x7f807f80u) + 0x00800080u);
      }
      if (__any_sync(0xffffffffu, hit & 0x80008000u)) {
#pragma unroll 1
        for (int key = 0; key < KEYS; ++key) {
          hit = 0;
          for (int w = lane; w < D / 2; w += 32)
            hit |= (*reinterpret_cast<const uint32_t *>(values + w / (PD / 2) * C::PART_BYTES + key * PB + w % (PD / 2) * 4) & 0x7f807f80u) + 0x00800080u;
          if (__any_sync(0xffffffffu, hit & 0x80008000u)) odd |= 1ull << key;
        }
      }
    }
    const uint32_t va = vst + wk * KEYS * PB + value_at;
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
      constexpr int GROUP = D / 16 < 4 ? D / 16 : 4;              // products of the high parts, then of the low parts: none waits for the one before
#pragma unroll
      for (int k0 = 0; k0 < D / 16; k0 += GROUP) {
        uint32_t v[GROUP][4];
#pragma unroll
        for (int j = 0; j < GROUP; ++j) {
          const int ks = k0 + j;
          flash_ldsm4_trans((va + n * 16 * PB + ks / (PD / 16) * C::PART_BYTES) ^ (uint32_t)(ks % (PD / 16) * 32), v[j]);
          if (odd) v[j][0] &= mask0, v[j][1] &= mask0, v[j][2] &= mask1, v[j][3] &= mask1;
        }
#pragma unroll
        for (int j = 0; j < GROUP; ++j)
#pragma unroll
          for (int q = 0; q < NQ; ++q) mma_bf16_16816(o[q][k0 + j], v[j], hi[q][0], hi[q][1]);
#pragma unroll
        for (int j = 0; j < GROUP; ++j)
#pragma unroll
          for (int q = 0; q < NQ; ++q) mma_bf16_16816(o[q][k0 + j], v[j], lo[q][0], lo[q][1]);
      }
      if (odd) {
#pragma unroll 1
        for (int key = 0; key < 16; ++key) {
          if (!(odd >> (n * 16 + key) & 1)) continue;
          const int slot = mine + n * 16 + key, row = wk * KEYS + n * 16 + key;
          const unsigned char *value = paged_smem + (vst - smem0) + row * PB;
#pragma unroll
          for (int q = 0; q < NQ; ++q)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const float p = __shfl_sync(0xffffffffu, key < 8 ? s[n][q][x] : s[n][q][2 + x], (key & 7) * 4 + t4);
              if (C::TREE ? !(sees(q, x) >> (n * 16 + key) & 1) : slot < range[q][x].x || slot >= range[q][x].y) continue;
#pragma unroll
              for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  o[q][ks][2 * e + x] = fmaf(p, to_f32(*reinterpret_cast<const bf16 *>(value + ks / (PD / 16) * C::PART_BYTES + flash_swz<PD>(row, (2 * ks + e) % (PD / 8)) * 16 + g * 2)), o[q][ks][2 * e + x]);
            }
        }
      }
    }

    if (it.t + 1 == tiles || i + 1 == run.count) {
      // the unit, or this CTA's part of it, ends: the other warps' parts through this stage's memory, in the fragments' order
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if (TMA && sh.dead) l[q][x] = NAN;
          l[q][x] += __shfl_xor_sync(0xffffffffu, l[q][x], 4);
          l[q][x] += __shfl_xor_sync(0xffffffffu, l[q][x], 8);
          l[q][x] += __shfl_xor_sync(0xffffffffu, l[q][x], 16);
        }
      if (WK > 1) {
        bar_sync(MERGE, 32 * C::WARPS);
        float4 *scratch = reinterpret_cast<float4 *>(paged_smem + stage * C::STAGE_BYTES) + lane;
        constexpr int WORDS = 32 * C::MERGE_WORDS;
        if (wk) {
          scratch += (wr * (WK - 1) + wk - 1) * WORDS;
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            scratch[32 * q] = make_float4(m[q][0], m[q][1], l[q][0], l[q][1]);
#pragma unroll
            for (int n = 0; n < D / 16; ++n) scratch[32 * (NQ + q * (D / 16) + n)] = make_float4(o[q][n][0], o[q][n][1], o[q][n][2], o[q][n][3]);
          }
        }
        bar_sync(MERGE, 32 * C::WARPS);
        if (!wk) {
#pragma unroll 1
          for (int w = 0; w < WK - 1; ++w) {
            const float4 *src = scratch + (wr * (WK - 1) + w) * WORDS;
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
              const float4 ml = src[32 * q];
              const float top0 = fmaxf(m[q][0], ml.x), top1 = fmaxf(m[q][1], ml.y);
              const float ref0 = top0 == -INFINITY ? 0.f : top0, ref1 = top1 == -INFINITY ? 0.f : top1;
              const float a0 = exp2f(m[q][0] - ref0), a1 = exp2f(m[q][1] - ref1), b0 = exp2f(ml.x - ref0), b1 = exp2f(ml.y - ref1);
              m[q][0] = top0, m[q][1] = top1;
              l[q][0] = l[q][0] * a0 + ml.z * b0, l[q][1] = l[q][1] * a1 + ml.w * b1;
#pragma unroll
              for (int n = 0; n < D / 16; ++n) {
                const float4 v = src[32 * (NQ + q * (D / 16) + n)];
                o[q][n][0] = o[q][n][0] * a0 + v.x * b0, o[q][n][1] = o[q][n][1] * a1 + v.y * b1;
                o[q][n][2] = o[q][n][2] * a0 + v.z * b0, o[q][n][3] = o[q][n][3] * a1 + v.w * b1;
              }
            }
          }
        }
      }
      if (!wk) {
        const int first_row = row0 + wr * WROWS;
        if (seg_first == 0 && it.t + 1 == tiles) {
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            const float inv0 = l[q][0] == 0.f ? 0.f : 1.f / l[q][0], inv1 = l[q][1] == 0.f ? 0.f : 1.f / l[q][1];
            const int row = first_row + q * 8 + g;         // after the transposition: query g, elements 2 t4, 2 t4 + 1 (+ 8)
            const bool live = row < R && token_of(a, row) < n_new;
            bf16 *out = live ? paged_out_row<bf16>(a, it.b, h, row, D) + t4 * 2 : nullptr;
#pragma unroll
            for (int n = 0; n < D / 16; ++n)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                // (an empty row's sums are 0, and 0 x inf cannot arise)
                const uint32_t y = movmatrix_trans(pack_bf16x2(o[q][n][2 * e] * inv0, o[q][n][2 * e + 1] * inv1));
                if (live) *reinterpret_cast<uint32_t *>(out + n * 16 + e * 8) = y;
              }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int r = first_row + q * 8 + t4 * 2 + x;
              if (g == 0 && r < R && token_of(a, r) < n_new) paged_write_lse(a, it.b, h, r, m[q][x], l[q][x]);
            }
          }
        } else {
          const int part = 2 * blockIdx.x + (seg_first == 0);
#pragma unroll
          for (int q = 0; q < NQ; ++q)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int r = wr * WROWS + q * 8 + t4 * 2 + x;
              if (row0 + r >= R) continue;
              float *dst = a.part_o + ((long long)part * ROWS + r) * D + g;
#pragma unroll
              for (int n = 0; n < D / 16; ++n) dst[n * 16] = o[q][n][x], dst[n * 16 + 8] = o[q][n][2 + x];
              if (g == 0) a.part_ml[part * ROWS + r] = make_float2(m[q][x], l[q][x]);
            }
        }
      }
    }
    if (i + S < run.count) {
      if (TMA) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");        // zeros and sums that were written here, before the next tile
      bar_arrive(EMPTY + stage, C::THREADS);
    }
    if (++stage == S) stage = 0;
  }
}

}  // namespace tsfm
