// The bf16 kernel of tsfm_paged_attention (work split and join: attn_paged.cuh): tiles of 64 slots in shared memory, products on
// mma.sync m16n8k16.
//
// WR x WK warps: a warp takes 16 query rows against 64 / WK of a tile's slots, with a running maximum and sum of its own; the WK
// warps of a row are merged when the unit ends.  Tiles (and the queries of a unit's first one) come in by cp.async, STAGES - 1
// tiles ahead and across unit borders, through a ring whose entries hold the byte offset of each slot's row: a page
// lookup a slot, not one a copy.  Precision: scores of bf16 operands in fp32; probabilities as two bf16 parts, so that only
// the result is rounded.
#pragma once
#include "attn_flash.cuh"
#include "attn_paged.cuh"

namespace tsfm {

template <int D, int WR> struct PagedMma {
  static constexpr int WK = 4 / WR, KEYS = PA_TILE / WK, BLOCKS = KEYS / 16;
  static constexpr int ROWS = 16 * WR, RB = D * 2;
  static constexpr int KV_BYTES = PA_TILE * RB, Q_BYTES = ROWS * RB, STAGE_BYTES = 2 * KV_BYTES + Q_BYTES;
  static constexpr int STAGES = D == 128 ? (WR == 1 ? 3 : 2) : D == 64 ? (WR == 1 ? 4 : 3) : 4;
  static constexpr int RING = STAGES + 1;
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES;
  // resident CTAs on an SM: beside the stages the ring, the scan (128 bytes), alignment, and 1 KB that a CTA costs; small
  // heads are bound by registers instead
  static constexpr int BY_SMEM = 228 * 1024 / (SMEM_BYTES + RING * (PA_TILE * 8 + 24) + 128 + 256 + 1024);
  static constexpr int CTAS = D == 32 ? (WR == 4 ? 3 : 4) : BY_SMEM;
  static_assert(4 * 16 * (D * 4 + 8) <= STAGE_BYTES, "the merge takes one stage");
};

// A tile on its way: unit u of series b, its t-th tile; b < 0: behind the run's end.
struct PagedItem {
  int b, u, t, first;                              // first: its queries come with it
};

template <int D, int WR>
__global__ void __launch_bounds__(PA_THREADS, PagedMma<D, WR>::CTAS) paged_attn_mma_kernel(const __grid_constant__ PagedAttnArgs a) {
  using C = PagedMma<D, WR>;
  constexpr int WK = C::WK, KEYS = C::KEYS, NB = C::BLOCKS, ROWS = C::ROWS, RB = C::RB, S = C::STAGES, RING = C::RING;
  constexpr int CPR = D / 8;                       // 16-byte chunks of a row
  extern __shared__ __align__(256) unsigned char paged_smem[];
  __shared__ long long s_off[RING][PA_TILE];       // byte offset of a slot's row in k and v, -1: hidden
  __shared__ unsigned s_valid[RING][2];
  __shared__ PagedItem s_item[RING];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wr = warp / WK, wk = warp % WK;
  const int g = lane >> 2, t4 = lane & 3;
  const uint32_t smem0 = (uint32_t)__cvta_generic_to_shared(paged_smem);
  const int R = a.M * a.group;
  const PagedRun run = paged_find_run<PA_THREADS>(a);
  if (tid == 0) {
    PagedMeta meta{-1, 0, 0, 0};
    if (run.count > 0 && run.first) {
      const int tiles = paged_span(a, run.b, false).tiles;
      meta = PagedMeta{run.b, run.u, (int)(run.unit0 / run.per), (int)((run.unit0 + tiles - 1) / run.per)};
    }
    a.meta[blockIdx.x] = meta;
  }
  if (run.count == 0) return;

  // the item that is looked up next, the same in every thread
  int nb = run.b, nu = run.u, nt = run.first, ni = 0;
  PagedSpan ns = paged_span(a, nb, false);
  auto look_up = [&](int slot_of_ring) {           // offsets of the next item; then moves on
    if (ni < run.count) {
      const int h = nu / a.chunks;
      if (tid < PA_TILE) {
        const int slot = (ns.tile0 + nt) * PA_TILE + tid;
        long long off = -1;
        if (slot >= ns.lo && slot < ns.total) {
          const int page = page_of(a.pg, a.pg.table + (long long)nb * a.pg.table_stride, slot);
          if (page >= 0) off = slot_offset(a.pg, page, h, slot);
          else pages_report(a.pg, BAD_ID);
        }
        s_off[slot_of_ring][tid] = off;
        const unsigned valid = __ballot_sync(0xffffffffu, off >= 0);
        if (lane == 0) s_valid[slot_of_ring][warp] = valid;
      }
      if (tid == 0) s_item[slot_of_ring] = PagedItem{nb, nu, nt, ni == 0 || nt == 0};
      ++ni;
      if (++nt == ns.tiles) {
        nt = 0;
        if (++nu == a.units) {
          nu = 0;
          while (ni < run.count) {                 // the next series that has tiles
            ns = paged_span(a, ++nb, false);
            if (ns.tiles) break;
          }
        }
      }
    } else if (tid == 0) {
      s_item[slot_of_ring].b = -1;
    }
  };
  const int cp_chunk = tid % CPR, cp_row = tid / CPR;
  auto load = [&](int slot_of_ring, int stage) {
    const PagedItem it = s_item[slot_of_ring];
    if (it.b >= 0) {
      const uint32_t dst = smem0 + stage * C::STAGE_BYTES;
#pragma unroll
      for (int r = cp_row; r < PA_TILE; r += PA_THREADS / CPR) {
        const long long off = s_off[slot_of_ring][r];
        const uint32_t at = dst + r * RB + flash_swz<D>(r, cp_chunk) * 16;
        const long long from = (off < 0 ? 0 : off) + cp_chunk * 16;
        const int bytes = off < 0 ? 0 : 16;        // hidden slots read as zeros
        asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(at), "l"(a.pg.k + from), "r"(bytes) : "memory");
        asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(at + C::KV_BYTES), "l"(a.pg.v + from), "r"(bytes) : "memory");
      }
      if (it.first) {
        const int h = it.u / a.chunks, row0 = (it.u - h * a.chunks) * ROWS;
#pragma unroll
        for (int r = cp_row; r < ROWS; r += PA_THREADS / CPR) {
          const bool in = row0 + r < R;
          const int tok = in ? (row0 + r) / a.group : 0, head = h * a.group + (in ? row0 + r - tok * a.group : 0);
          const bf16 *src = reinterpret_cast<const bf16 *>(a.q) + ((long long)it.b * a.M + tok) * a.q_stride + (long long)head * D + cp_chunk * 8;
          const uint32_t at = dst + 2 * C::KV_BYTES + r * RB + flash_swz<D>(r, cp_chunk) * 16;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(src), "r"(in ? 16 : 0) : "memory");
        }
      }
    }
    flash_commit();
  };

  for (int j = 0; j < S; ++j) look_up(j);
  __syncthreads();
  for (int j = 0; j < S - 1; ++j) load(j, j);

  const FlashLane<D> fl(lane);
  uint32_t qf[D / 16][4];
  float o[D / 8][4], m[2], l[2];
  int2 range[2];                                   // what rows g and g + 8 see
  int min_end = 0, max_start = 0, total = 0, tile0 = 0, tiles = 0, len_lo = 0, seg_first = 0, n_new = 0, h = 0, row0 = 0;
  for (int i = 0; i < run.count; ++i) {
    const int stage = i % S, ring = i % RING;
    flash_wait<S - 2>();
    __syncthreads();
    load((i + S - 1) % RING, (i + S - 1) % S);
    look_up((i + S) % RING);
    const PagedItem it = s_item[ring];
    const uint32_t kst = smem0 + stage * C::STAGE_BYTES, vst = kst + C::KV_BYTES;
    if (it.first) {
      const PagedSpan s = paged_span(a, it.b, false);
      h = it.u / a.chunks, row0 = (it.u - h * a.chunks) * ROWS;
      total = s.total, tile0 = s.tile0, tiles = s.tiles, len_lo = s.lo, n_new = s.n_new, seg_first = it.t;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int row = row0 + wr * 16 + g + 8 * x;
        range[x] = row < R ? paged_row_range(a, s, row / a.group) : make_int2(0, 0);
        m[x] = -INFINITY;
        l[x] = 0.f;
      }
      min_end = paged_row_range(a, s, row0 / a.group).y;
      max_start = paged_row_range(a, s, min(s.n_new, (min(R, row0 + ROWS) - 1) / a.group + 1) - 1).x;
      const int qrow = wr * 16 + (lane & 15);
      const uint32_t qa = vst + C::KV_BYTES + qrow * RB + flash_swz<D>(qrow, lane >> 4) * 16;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) flash_ldsm4(qa ^ (uint32_t)(ks * 32), qf[ks]);
#pragma unroll
      for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    }
    const int base = (tile0 + it.t) * PA_TILE, mine = base + wk * KEYS;       // slots of the tile, of this warp
    const unsigned long long valid = s_valid[ring][0] | (unsigned long long)s_valid[ring][1] << 32;

    // scores
    float s[NB][2][4];
    const uint32_t ka = kst + wk * KEYS * RB + fl.ka;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
#pragma unroll
      for (int x = 0; x < 4; ++x) s[n][0][x] = s[n][1][x] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        uint32_t b[4];
        flash_ldsm4((ka + n * 16 * RB) ^ (uint32_t)(ks * 32), b);
        mma_bf16_16816(s[n][0], qf[ks], b[0], b[1]);
        mma_bf16_16816(s[n][1], qf[ks], b[2], b[3]);
      }
    }
    const bool open = valid == ~0ull && base >= max_start && base + PA_TILE <= min_end;      // every row sees every slot
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[n][e][x] *= a.scale2;
    if (!open) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int at = n * 16 + e * 8 + t4 * 2 + (x & 1), slot = mine + at;
            const int2 r = range[x >> 1];
            if (slot < r.x || slot >= r.y || !(valid >> (wk * KEYS + at) & 1)) s[n][e][x] = -INFINITY;
          }
    }
    if (a.scores) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int row = row0 + wr * 16 + g + 8 * x;
        if (row >= R) continue;
        float *dst = a.scores + (((long long)it.b * a.pg.n_kv_heads + h) * R + row) * a.score_stride + mine + t4 * 2;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (mine + n * 16 + e * 8 + t4 * 2 < total) *reinterpret_cast<float2 *>(dst + n * 16 + e * 8) = make_float2(s[n][e][2 * x], s[n][e][2 * x + 1]);
      }
    }
    // running softmax of rows g and g + 8
    float alpha[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float top = m[x];
#pragma unroll
      for (int n = 0; n < NB; ++n) top = fmaxf(top, fmaxf(fmaxf(s[n][0][2 * x], s[n][0][2 * x + 1]), fmaxf(s[n][1][2 * x], s[n][1][2 * x + 1])));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float ref = top == -INFINITY ? 0.f : top;
      alpha[x] = flash_ex2(m[x] - ref);
      m[x] = top;
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          s[n][e][2 * x] = flash_ex2(s[n][e][2 * x] - ref);
          s[n][e][2 * x + 1] = flash_ex2(s[n][e][2 * x + 1] - ref);
          sum += s[n][e][2 * x] + s[n][e][2 * x + 1];
        }
      l[x] = fmaf(l[x], alpha[x], sum);
    }
#pragma unroll
    for (int n = 0; n < D / 8; ++n) o[n][0] *= alpha[0], o[n][1] *= alpha[0], o[n][2] *= alpha[1], o[n][3] *= alpha[1];

    // Where some rows see a slot and others do not, a value that is not finite must not reach the others as 0 x NaN: such
    // slots (rare) leave the products and are added to the rows that see them.
    unsigned long long odd = 0;
    const int from = max(mine, len_lo), to = min(mine + KEYS, total);
    if (a.M > 1 && (max(from, min_end) < to || from < min(to, max_start))) {
      for (int key = 0; key < KEYS; ++key) {
        constexpr int WORDS = D / 64 > 0 ? D / 64 : 1;                        // 32-bit words a lane looks at
        const unsigned char *row = paged_smem + (vst - smem0) + (wk * KEYS + key) * RB;
        bool bad = false;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
          if (lane + 32 * w < D / 2) {
            const uint32_t v = reinterpret_cast<const uint32_t *>(row)[lane + 32 * w];
            bad |= (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u;
          }
        }
        if (__any_sync(0xffffffffu, bad)) odd |= 1ull << key;
      }
    }
    const uint32_t va = vst + wk * KEYS * RB + fl.va;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      uint32_t hi[4], lo[4];                       // a fragment of P: rows g, g + 8; slots 2 t4 (+ 8)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const float p0 = s[n][y >> 1][2 * (y & 1)], p1 = s[n][y >> 1][2 * (y & 1) + 1];
        hi[y] = pack_bf16x2(p0, p1);
        lo[y] = pack_bf16x2(p0 - __uint_as_float(hi[y] << 16), p1 - __uint_as_float(hi[y] & 0xffff0000u));
      }
      uint32_t mask0 = ~0u, mask1 = ~0u;
      if (odd) {
        const unsigned bits = (unsigned)(odd >> (n * 16)) >> (2 * t4);
        mask0 = (bits & 1 ? 0u : 0xffffu) | (bits & 2 ? 0u : 0xffff0000u);
        mask1 = (bits & 256 ? 0u : 0xffffu) | (bits & 512 ? 0u : 0xffff0000u);
      }
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        uint32_t b[4];
        flash_ldsm4_trans((va + n * 16 * RB) ^ (uint32_t)(ks * 32), b);
        if (odd) b[0] &= mask0, b[1] &= mask1, b[2] &= mask0, b[3] &= mask1;
        mma_bf16_16816(o[2 * ks], hi, b[0], b[1]);
        mma_bf16_16816(o[2 * ks + 1], hi, b[2], b[3]);
        mma_bf16_16816(o[2 * ks], lo, b[0], b[1]);
        mma_bf16_16816(o[2 * ks + 1], lo, b[2], b[3]);
      }
      if (odd) {
#pragma unroll 1
        for (int key = 0; key < 16; ++key) {
          if (!(odd >> (n * 16 + key) & 1)) continue;
          const int slot = mine + n * 16 + key, row = wk * KEYS + n * 16 + key;
          float p[2];                              // this slot's probability for rows g and g + 8
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float even = key < 8 ? s[n][0][2 * x] : s[n][1][2 * x], odd_ = key < 8 ? s[n][0][2 * x + 1] : s[n][1][2 * x + 1];
            p[x] = __shfl_sync(0xffffffffu, key & 1 ? odd_ : even, (lane & ~3) | ((key & 7) >> 1));
          }
#pragma unroll
          for (int d = 0; d < D / 8; ++d) {
            const uint32_t v = *reinterpret_cast<const uint32_t *>(paged_smem + (vst - smem0) + row * RB + flash_swz<D>(row, d) * 16 + t4 * 4);
            const float v0 = __uint_as_float(v << 16), v1 = __uint_as_float(v & 0xffff0000u);
#pragma unroll
            for (int x = 0; x < 2; ++x)
              if (slot >= range[x].x && slot < range[x].y) o[d][2 * x] = fmaf(p[x], v0, o[d][2 * x]), o[d][2 * x + 1] = fmaf(p[x], v1, o[d][2 * x + 1]);
          }
        }
      }
    }

    if (it.t + 1 == tiles || i + 1 == run.count) {
      // the unit, or this CTA's part of it, ends: all warps' parts through this stage's memory, then the result by all threads
      const int rows = min(ROWS, R - row0);
      __syncthreads();
      float *scratch = reinterpret_cast<float *>(paged_smem + stage * C::STAGE_BYTES);        // [warp][16][D]
      float2 *ml_scratch = reinterpret_cast<float2 *>(scratch + 4 * 16 * D);                  // [warp][16]
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = g + 8 * x;
        l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
        l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
        if (wr * 16 + r < rows) {
          if (t4 == 0) ml_scratch[warp * 16 + r] = make_float2(m[x], l[x]);
#pragma unroll
          for (int n = 0; n < D / 8; ++n)
            *reinterpret_cast<float2 *>(scratch + (warp * 16 + r) * D + n * 8 + t4 * 2) = make_float2(o[n][2 * x], o[n][2 * x + 1]);
        }
      }
      __syncthreads();
      const bool whole = seg_first == 0 && it.t + 1 == tiles;
      const int part = 2 * blockIdx.x + (seg_first == 0);
      for (int e = tid; e < rows * (D / 4); e += PA_THREADS) {
        const int r = e / (D / 4), d = (e - r * (D / 4)) * 4, w0 = (r >> 4) * WK, rl = r & 15;
        float top = ml_scratch[w0 * 16 + rl].x;
#pragma unroll
        for (int w = 1; w < WK; ++w) top = fmaxf(top, ml_scratch[(w0 + w) * 16 + rl].x);
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WK; ++w) {
          const float2 ml = ml_scratch[(w0 + w) * 16 + rl];
          const float f = exp2f(ml.x - ref);
          const float4 x = *reinterpret_cast<const float4 *>(scratch + ((w0 + w) * 16 + rl) * D + d);
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
  }
  flash_wait<0>();
}

}  // namespace tsfm
