// How tiles of slots come into shared memory for the kernels of tsfm_paged_attention: one warp of a CTA looks pages up, copies, waits
// for the copies and hands the stages over by named barriers; the other warps compute.
//
// A tile is 64 slots of one key head: keys, then values, each as parts of 128-byte (64-byte) rows, [part][slot], whose 16-byte chunks are
// exchanged as TMA's swizzle does; behind them the queries of a unit's first tile.  TMA copies boxes of up to 64 slots of a page; pages of
// less than eight slots, and pools that the driver makes no map for, go by cp.async, a slot's row at a time.
#pragma once
#include <climits>
#include "attn_flash.cuh"
#include "attn_paged.cuh"
#include "gemm_tc.cuh"

namespace tsfm {

// Barriers between the fetching warp and the others: `full` of a stage, `empty` of a stage; and one among the others.
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__host__ __device__ constexpr int bar_full() { return 1; }
__host__ __device__ constexpr int bar_empty(int stages) { return 1 + stages; }
__host__ __device__ constexpr int bar_merge(int stages) { return 1 + 2 * stages; }

// Place of chunk c of a slot's row of PB bytes; of a query's row of RB bytes.
template <int PB> __device__ __forceinline__ int tile_swz(int r, int c) { return PB == 64 ? c ^ ((r >> 1) & 3) : c ^ (r & 7); }
template <int RB> __device__ __forceinline__ int query_swz(int r, int c) { return tile_swz<RB>(r, c); }

// A tile on its way: unit u of series b, its t-th tile, and the series' span.  first: the unit's queries come with it.
struct PagedItem {
  int b, u, t, first;
  PagedSpan sp;
};

// TMA tile of a page's slots: {first element, slot, head, page}.
__device__ __forceinline__ void tma_load_page(uint32_t dst, const CUtensorMap *map, int x, int slot, int head, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(x), "r"(slot), "r"(head), "r"(page), "r"(bar) : "memory");
}
// Bounded wait for a tile: false if it did not arrive within `limit` ns.
__device__ __forceinline__ bool tile_arrived(uint32_t bar, uint32_t parity, unsigned long long limit) {
  unsigned long long t0 = 0;
  for (uint32_t n = 0;; ++n) {
    if (mbar_try_wait(bar, parity)) return true;
    if (n == 256) t0 = globaltimer_ns();
    if (n > 256 && (n & 255) == 0 && globaltimer_ns() - t0 > limit) return false;
  }
}

// What describes the stages, beside them.
template <int S, bool TMA> struct PagedStages {
  unsigned long long full[S];                      // TMA's barriers, waited on by the fetching warp alone
  unsigned valid[S][2];                            // slots of the tile that exist: in [lo, total), page in the pool
  PagedItem item[S], next[S];                      // of the stages; of the tiles whose page ids are on their way
  int ids[S][TMA ? 8 : PA_TILE];                   // those ids
  int dead;                                        // a tile did not arrive: what is computed from here on is NaN
};

// C: D, RB (bytes of a slot's row), PD, PB, PARTS, PART_BYTES, KV_BYTES, ROWS, STAGES, STAGE_BYTES, THREADS.
template <typename C, bool TMA>
__device__ __forceinline__ void paged_fetch(const PagedAttnArgs &a, const PagedRun &run, PagedStages<C::STAGES, TMA> &sh, uint32_t smem0, const CUtensorMap &mapK,
                                            const CUtensorMap &mapV) {
  constexpr int S = C::STAGES, FULL = bar_full(), EMPTY = bar_empty(S), ROWS = C::ROWS, PB = C::PB, PARTS = C::PARTS;
  const int lane = threadIdx.x & 31, R = a.M * a.group;
  constexpr int CPR = C::RB / 16, STEP = 32 / CPR;       // 16-byte chunks of a row; rows of a copy instruction
  const int chunk = lane % CPR, sub = lane / CPR;
  // Page ids travel like the tiles, AHEAD tiles before theirs and in the same groups: a plain load behind the queue of copies
  // returned after 6000 to 17000 cycles and stood between each tile and the next.
  constexpr int AHEAD = S - 1;
  int b = run.b, u = run.u, t = run.first, ni = 0;
  PagedSpan sp = paged_span(a, b, false);
  int len_next = 0, new_next = 0;                // of series b + 1, looked at when it is reached
  auto fetch_next = [&]() {
    const int at = min(b + 1, a.B - 1);
    len_next = __ldg(a.len + at);
    new_next = a.n_new ? __ldg(a.n_new + at) : a.M;
  };
  fetch_next();
  // TMA copies boxes of up to 64 slots of one page: a page id a box, else a slot
  const int box_log = TMA ? min(a.pg.page_log, 6) : 0, boxes = PA_TILE >> box_log;
  const uint32_t full0 = smem_u32(sh.full);
  bool dead = false;                             // a tile did not arrive: nothing more is fetched
  int late = 0, issued = INT_MAX;                // (TMA) that tile; the last one that had been asked for by then
  if (lane == 0) sh.dead = 0;
  if (TMA) {
    if (lane < S) mbar_init(full0 + 8 * lane, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
  }
  auto fetch_ids = [&]() {                       // of tile ni; then moves on
    if (ni >= run.count) return;
    const int ring = ni % S;
    const int *row = a.pg.table + (long long)b * a.pg.table_stride;
#pragma unroll
    for (int x = 0; x < (TMA ? 1 : 2); ++x) {
      const int j = 32 * x + lane, slot = (sp.tile0 + t) * PA_TILE + (j << box_log);
      if (j < boxes && slot + (1 << box_log) > sp.lo && slot < sp.total)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(&sh.ids[ring][j])), "l"(row + (slot >> a.pg.page_log)) : "memory");
    }
    if (lane == 0) sh.next[ring] = PagedItem{b, u, t, ni == 0 || t == 0, sp};
    if (++ni == run.count) return;
    paged_next_tile(b, u, t, sp, a.B, a.units, [&]() {
      const PagedSpan at = paged_span_of(a, len_next, new_next, false);
      fetch_next();
      return at;
    });
  };
  for (int j = 0; j < AHEAD; ++j) fetch_ids();
  flash_commit();
  flash_wait<0>();
  int stage = 0;
  for (int i = 0; i < run.count; ++i) {
    const uint32_t dst = smem0 + stage * C::STAGE_BYTES;
    __syncwarp();
    const PagedItem it = sh.next[stage];
    const int h = it.u / a.chunks;
    const int base = (it.sp.tile0 + it.t) * PA_TILE;
    long long off[2] = {-1, -1};                 // (plain copies) byte offsets of slots lane, lane + 32; -1: hidden
    int page = -1;                               // (TMA) of box lane % 8
    unsigned v[2];
    if (TMA) {
      const int j = lane & 7, slot = base + (j << box_log);
      if (j < boxes && slot + (1 << box_log) > it.sp.lo && slot < it.sp.total) {
        page = sh.ids[stage][j];
        if ((unsigned)page >= (unsigned)a.pg.n_pages) {
          page = -1;
          pages_report(a.pg, BAD_ID);
        }
      }
      const unsigned ok = __ballot_sync(0xffffffffu, page >= 0) & 0xff;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int at = 32 * x + lane;
        v[x] = __ballot_sync(0xffffffffu, base + at >= it.sp.lo && base + at < it.sp.total && (ok >> (at >> box_log) & 1));
      }
    } else {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int slot = base + 32 * x + lane;
        if (slot >= it.sp.lo && slot < it.sp.total) {
          const int id = sh.ids[stage][32 * x + lane];
          if ((unsigned)id < (unsigned)a.pg.n_pages) off[x] = slot_offset(a.pg, id, h, slot);
          else pages_report(a.pg, BAD_ID);
        }
        v[x] = __ballot_sync(0xffffffffu, off[x] >= 0);
      }
    }
    __syncwarp();
    fetch_ids();
    if (i >= S) bar_sync(EMPTY + stage, C::THREADS);
    if (lane == 0) {
      sh.valid[stage][0] = v[0], sh.valid[stage][1] = v[1];
      sh.item[stage] = it;
    }
    if (TMA) {
      const unsigned ok = __ballot_sync(0xffffffffu, page >= 0) & 0xff;
      if (lane == 0 && !dead) mbar_expect_tx(full0 + 8 * stage, __popc(ok) * 2 * PARTS * (PB << box_log) + (i >= a.miss_from ? 16 : 0));
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 16 * PARTS; i += 32) {   // (box, part, keys or values)
        const int part = ((i + lane) >> 3) % PARTS, kv = ((i + lane) >> 3) / PARTS;
        if (page >= 0 && kv < 2 && !dead) {
          const int slot = base + ((lane & 7) << box_log);
          tma_load_page(dst + kv * C::KV_BYTES + part * C::PART_BYTES + ((lane & 7) << box_log) * PB, kv ? &mapV : &mapK, part * C::PD,
                        slot & ((1 << a.pg.page_log) - 1), h, page, full0 + 8 * stage);
        }
      }
    } else {
#pragma unroll
      for (int r = 0; r < PA_TILE; r += STEP) {
        const long long o = __shfl_sync(0xffffffffu, off[r / 32], (r & 31) + sub);
        const uint32_t at = dst + chunk / (PB / 16) * C::PART_BYTES + (r + sub) * PB + tile_swz<PB>(r + sub, chunk % (PB / 16)) * 16;
        const long long from = (o < 0 ? 0 : o) + chunk * 16;
        const int bytes = o < 0 ? 0 : 16;        // hidden slots arrive as zeros
        asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(at), "l"(a.pg.k + from), "r"(bytes) : "memory");
        asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(at + C::KV_BYTES), "l"(a.pg.v + from), "r"(bytes) : "memory");
      }
    }
    if (it.first) {
      const int row0 = (it.u - h * a.chunks) * ROWS;
#pragma unroll 4
      for (int r = sub; r < ROWS; r += STEP) {
        const bool in = row0 + r < R;
        const int tok = in ? token_of(a, row0 + r) : 0, head = h * a.group + (in ? row0 + r - tok * a.group : 0);
        const char *src = reinterpret_cast<const char *>(a.q) + (((long long)it.b * a.M + tok) * a.q_stride + (long long)head * C::D) * (C::RB / C::D) + chunk * 16;
        const uint32_t at = dst + 2 * C::KV_BYTES + r * C::RB + query_swz<C::RB>(r, chunk) * 16;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(src), "r"(in ? 16 : 0) : "memory");
      }
    }
    flash_commit();
    auto hand_over = [&](int tile) {
      // (tiles that were on their way when one did not arrive are waited for too)
      if (TMA && tile <= issued && __any_sync(0xffffffffu, !tile_arrived(full0 + 8 * (tile % S), (tile / S) & 1, a.wait_ns))) {
        if (!dead) late = tile, issued = i;
        dead = true;
        if (lane == 0) sh.dead = 1;
        pages_report(a.pg, PAGES_TIMEOUT);
      }
      __threadfence_block();
      bar_arrive(FULL + tile % S, C::THREADS);
    };
    if (i >= S - 2) {
      flash_wait<S - 2>();
      hand_over(i - (S - 2));
    }
    if (i + 1 == run.count) {
      flash_wait<0>();
      for (int tile = max(0, run.count - (S - 2)); tile < run.count; ++tile) hand_over(tile);
    }
    if (++stage == S) stage = 0;
  }
  // No copy may land in shared memory that is no longer this CTA's: those that gave no sign get another limit each.
  if (TMA && dead)
    for (int tile = late; tile <= issued; ++tile) tile_arrived(full0 + 8 * (tile % S), (tile / S) & 1, a.wait_ns);
}

}  // namespace tsfm
