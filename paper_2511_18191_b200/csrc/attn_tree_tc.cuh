// Attention of many rows over a cache of pages (trees of some dozens of nodes, prompts; masks of attn_tree.cuh) on the tensor cores:
// tcgen05, bf16, heads of 64 and 128, pages of eight slots and more.
//
// A CTA takes a run of tiles as in attn_paged.cuh, of units of QT x 128 rows (new tokens x the heads of a group).  A tile is two blocks of 64 slots,
// wherever in the cache they lie (a block with sinks beside one of the window).  Of each, for 128 rows at a time:
//   S = Q K^T (128 x 128, queries and keys as they are: products of bf16, sums in fp32, in tensor memory); softmax by two threads a row, each
//   the slots of one block: exponentials, sum, maximum; P back over S as two bf16 parts, the high and the low ones of 16 slots in the columns that held
//   their scores; O += P V in tensor memory, both parts.
// Softmax is the same whatever is subtracted from the scores, as long as nothing overflows and the largest terms do not vanish.  So the exponentials
// do not wait for the row's maximum: they are taken against a reference, 2^20 at first, and where the maximum of the next 16 slots turns out to lie above it (the first
// one: or 2^40 below) the reference moves 2^20 above that.  References are whole numbers, so what was there before follows by products with powers of two, which are
// exact: the tile's probabilities at its end, O in tensor memory.  With scores of ordinary size that never happens, and O is read once, when the unit ends.
// No exponential is above 1, so sums overflow where those of another kernel would; what of a result lies below 2^-80 may be lost.
// QT = 1: two CTAs on an SM, one's products run beside the other's softmax.  QT = 2: one CTA with two times 128 rows, which share the tiles that
// they read and take turns in the same way.
// A slot that some row must not see never meets it as 0 x NaN: values outside the series' slots are zeroed in shared memory; in tiles that not every
// row sees as a whole, elements that are not finite are zeroed too, and rows that do see one get NaN in its column, and there alone.
// Precision: as paged_attn_mma_kernel: 2^-16 of a probability is lost (P in two bf16 parts; with one, 2^-8, the output was off by 0.0023 of its norm where its own
// rounding is 0.0017), sums are fp32 and of the unrounded exponentials.  The second part is half as much work again for the tensor core.
// Bound: the chain of a tile's softmax (2900 cycles for 64 slots a thread, beside 1536 of products; tensor pipe 45 %, issue 0.43 a cycle).  32 series of up to 8192
// slots, 61 nodes x 4 heads of 128 a key head: 229 us and 20 of the join, 460 TFLOP/s of what the definition needs, 568 MB from DRAM (87 us); 4 prompts of up to 4096
// tokens in a window of 1024: 555 us and 19.  What was tried and slower: half of the exponentials by FMA, the maximum in a pass of its own, values looked at by the
// warp of the products, two groups of softmax warps on one stream of tiles; with two parts, 16 slots' maximum taken while those before are exponentiated (spills),
// code of its own for tiles without masks (tree-large 225 -> 216, window-prompts 540 -> 601).
// Warps 0 .. 8 QT - 1 softmax (row 32 (w % 4) + lane of 128, block w / 4 % 2), then one that fetches (TMA: boxes of a page, queries) and one for tensor
// memory and products.  Every wait is bounded; when one runs out the status says so and what depends on it is NaN.
#pragma once
#include "attn_mma.cuh"
#include "attn_paged_fetch.cuh"

namespace tsfm {

template <int D_, int QT_> struct TreeTc {
  static constexpr int D = D_, QT = QT_, ROWS = 128 * QT, RB = D * 2, PARTS = D / 64;
  static constexpr int PART_BYTES = 128 * 128;                   // 128 rows (slots, queries) of 64 elements
  static constexpr int TILE_BYTES = PARTS * PART_BYTES;
  static constexpr int STAGES = D == 128 && QT == 1 ? 1 : 2;     // of keys and of values
  static constexpr int SMEM_BYTES = (QT + 2 * STAGES) * TILE_BYTES + 1024;       // (queries first; parts begin at multiples of 1 KB)
  static constexpr int WARPS = 8 * QT, THREADS = 32 * (WARPS + 2), CTAS = 2 / QT;
  static constexpr int COLS = 256 * QT, O = 128 * QT;            // columns of tensor memory: scores, sums; probabilities lie over their scores
  static constexpr int START = 2;                                // what starts and ends a unit, in tiles
  static_assert(CTAS * (SMEM_BYTES + 9 * 1024 + 512) <= 228 * 1024, "CTAs on an SM");
};
constexpr float TREE_TC_SLACK = 20.f;              // powers of two between a row's maximum and its reference when that is set; up to twice as many later

struct TreeTcShared {
  unsigned long long kfull[2], kempty[2], vfull[2], vempty[2], info[4], taken[4], s_full[2], p_ready[2], o_full[2], looked[2], q_ready, drained;
  unsigned long long valid[4][2];                  // of a tile's blocks: slots that exist
  float top[2][2][128], sum[2][2][128];            // what the two threads of a row exchange
  uint32_t bad[4][2][4];                           // slots of such a tile with values that are not finite, in the first and the second half of the columns
  unsigned long long columns[2][128][2];           // which, of those slots
  uint32_t tmem;
  int dead;                                        // a wait ran out: what is stored from here on is NaN
};

// A CTA's way through its run; every role walks by itself.  Of the unit only what every tile asks for is kept: registers are short, and what the
// spilled ones cost in every tile was more than all else that is not softmax.
struct TreeWalk {
  int b, u, t;
  int blocks, sink, gap;                           // of the unit: its blocks, those with sinks, slots between these and the others
  __device__ __forceinline__ int tiles() const { return (blocks + 1) >> 1; }
  __device__ __forceinline__ PagedSpan span(const PagedAttnArgs &a, int rows) const { return paged_unit_span<2>(a, b, u / a.pg.n_kv_heads, rows, false); }
  __device__ __forceinline__ bool enter(const PagedAttnArgs &a, int rows) {        // false: the unit has no live row
    const PagedSpan s = span(a, rows);
    blocks = paged_unit_blocks(a, s);
    sink = paged_sink_tiles(a, s);
    gap = (s.tile0 - sink) * PA_TILE;
    return s.tiles;
  }
  __device__ __forceinline__ TreeWalk(const PagedAttnArgs &a, const PagedRun &run, int rows) : b(run.b), u(run.u), t(run.first) { enter(a, rows); }
  // (bounded by the series, as paged_next_tile is)
  __device__ __forceinline__ void next(const PagedAttnArgs &a, int rows) {
    if (++t < tiles()) return;
    t = 0;
    if (++u < a.units && (u % a.pg.n_kv_heads || enter(a, rows))) return;         // (another head's rows of the same chunk, or the next chunk)
    u = 0;
    while (b + 1 < a.B) {
      ++b;
      if (enter(a, rows)) break;
    }
  }
  // First slot of block x of the tile; whether the second is one.
  __device__ __forceinline__ int base(int x) const {
    const int k = 2 * t + x;
    return k * PA_TILE + (k < sink ? 0 : gap);
  }
  __device__ __forceinline__ bool two() const { return 2 * t + 1 < blocks; }
  // How many times 128 rows of the unit hold a live one.
  template <int QT> __device__ __forceinline__ int halves(const PagedAttnArgs &a, const PagedSpan &s) const {
    return QT == 2 && s.n_new * (long long)a.group - u / a.pg.n_kv_heads * (128ll * QT) > 128 ? 2 : 1;
  }
};

__device__ __forceinline__ void tmem_load16(uint32_t taddr, float (&v)[16]) {        // (tmem_wait16 behind it)
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
        "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(taddr) : "memory");
}
// (names the values: nothing that uses them moves in front of the wait)
__device__ __forceinline__ void tmem_wait16(float (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]),
                 "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
               :: "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tma_load_queries(uint32_t dst, const CUtensorMap *map, int x, int head, int token, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(x), "r"(head), "r"(token), "r"(bar) : "memory");
}
// Barrier of 64 threads that says whether any of them brought true.
__device__ __forceinline__ bool bar_any64(int id, bool mine) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any) : "r"((uint32_t)mine), "r"(id) : "memory");
  return any != 0;
}

// q_tma: mapQ is there (a group divides 128); else queries come by cp.async, a row at a time.
template <typename C>
__global__ void __launch_bounds__(C::THREADS, C::CTAS)
tree_attn_tc_kernel(const __grid_constant__ PagedAttnArgs a, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                    const __grid_constant__ CUtensorMap mapQ, int q_tma) {
  constexpr int D = C::D, ROWS = C::ROWS, ST = C::STAGES, PARTS = C::PARTS, QT = C::QT;
  extern __shared__ __align__(1024) unsigned char paged_smem_raw[];
  __shared__ TreeTcShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), Hkv = a.pg.n_kv_heads;
  const uint32_t smem0 = (smem_u32(paged_smem_raw) + 1023u) & ~1023u;
  unsigned char *const smem = paged_smem_raw + (smem0 - smem_u32(paged_smem_raw));
  const uint32_t keys0 = smem0 + QT * C::TILE_BYTES, values0 = keys0 + ST * C::TILE_BYTES;
  const uint32_t kfull = smem_u32(sh.kfull), kempty = smem_u32(sh.kempty), vfull = smem_u32(sh.vfull), vempty = smem_u32(sh.vempty), info = smem_u32(sh.info), taken = smem_u32(sh.taken);
  const uint32_t q_ready = smem_u32(&sh.q_ready), s_full = smem_u32(sh.s_full), p_ready = smem_u32(sh.p_ready), o_full = smem_u32(sh.o_full),
                 looked = smem_u32(sh.looked), drained = smem_u32(&sh.drained);
  const int R = a.M * a.group;
  const PagedRun run = paged_find_unit_run<C::THREADS, 2>(a, ROWS, C::START);
  pdl_release();                                   // (the join waits for this grid's end; its CTAs may take their places)
  if (tid == 0) {
    PagedMeta meta{-1, 0, 0, 0};
    if (run.count > 0 && run.first) {
      const int tiles = paged_unit_span<2>(a, run.b, run.u / Hkv, ROWS, false).tiles;
      meta = PagedMeta{run.b, run.u, (int)(run.unit0 / run.per), (int)min((run.unit0 + tiles - 1) / run.per, (long long)gridDim.x - 1)};
    }
    a.meta[blockIdx.x] = meta;
  }
  if (run.count == 0) return;
  const bool leader = elect_one();
  if (warp == C::WARPS) {
    if (lane < 2) {
      mbar_init(kfull + 8 * lane, 1);
      mbar_init(kempty + 8 * lane, 1);
      mbar_init(vfull + 8 * lane, 1);
      mbar_init(vempty + 8 * lane, 1);
      mbar_init(s_full + 8 * lane, 1);
      mbar_init(p_ready + 8 * lane, 8);
      mbar_init(o_full + 8 * lane, 1);
      mbar_init(looked + 8 * lane, 8);
    }
    if (lane < 4) {
      mbar_init(info + 8 * lane, 1);
      mbar_init(taken + 8 * lane, C::WARPS);
    }
    (&sh.bad[0][0][0])[lane] = 0;
    if (lane == 0) {
      mbar_init(q_ready, 1);
      mbar_init(drained, 1);
      sh.dead = 0;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  } else if (warp == C::WARPS + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"((uint32_t)C::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  bool ok = true;
  int keys = 0, values = 0, queries = 0;           // (of the warp that fetches) copies that it has asked for
  // a bounded wait of a whole warp; one that ran out is reported, and there are no more
  auto wait = [&](uint32_t bar, int phase) {
    if (ok && __any_sync(0xffffffffu, !tile_arrived(bar, (uint32_t)phase & 1, a.wait_ns))) {
      ok = false;
      sh.dead = 1;
      pages_report(a.pg, PAGES_TIMEOUT);
    }
  };

  if (warp == C::WARPS) {
    // ---------------- fetches
    const int box_log = min(a.pg.page_log, 6), boxes = PA_TILE >> box_log;
    TreeWalk ahead(a, run, ROWS);                  // the tile whose page ids are looked up; lane 8 h + j: box j of block h
    PagedSpan span_ahead = ahead.span(a, ROWS);
    int id = 0;                                    // (not looked at before its tile's turn: nothing waits for the load until then)
    bool asked = false;
    int h = 0;
    auto look_up = [&]() {
      const int h = lane >> 3, j = lane & 7;
      asked = h < 2 && j < boxes && (h == 0 || ahead.two());
      const int slot = ahead.base(h) + (j << box_log);
      asked = asked && paged_wants<true>(a, span_ahead, slot, 1 << box_log);
      if (asked) id = __ldg(a.pg.table + (long long)ahead.b * a.pg.table_stride + (slot >> a.pg.page_log));
    };
    look_up();
    for (int i = 0; i < run.count && ok; ++i) {
      const int stage = i % ST, use = i / ST, page = asked && (unsigned)id < (unsigned)a.pg.n_pages ? id : -1;
      if (__any_sync(0xffffffffu, asked && page < 0)) pages_report(a.pg, BAD_ID);
      const TreeWalk at = ahead;
      const PagedSpan span = span_ahead;
      if (i + 1 < run.count) {
        ahead.next(a, ROWS);
        if (ahead.t == 0) span_ahead = ahead.span(a, ROWS);
        look_up();
      }
      const bool first = i == 0 || at.t == 0;
      const unsigned got = __ballot_sync(0xffffffffu, page >= 0);
      if (first) h = at.u % Hkv;
      const bool two = at.two();
      int base[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) base[x] = at.base(x);
      unsigned v[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int s = (x & 1) * 32 + lane;
        v[x] = __ballot_sync(0xffffffffu, (x < 2 || two) && paged_wants<true>(a, span, base[x >> 1] + s, 1) && (got >> ((x >> 1) * 8 + (s >> box_log)) & 1));
      }
      auto issue = [&](uint32_t dst, const CUtensorMap *map, uint32_t bar, int more) {
        if (lane == 0) mbar_expect_tx(bar, __popc(got) * (PARTS * 128 << box_log) + more);
        __syncwarp();
        if (page >= 0) {
          const int slot = (lane >> 3 ? base[1] : base[0]) + ((lane & 7) << box_log);
#pragma unroll
          for (int p = 0; p < PARTS; ++p)
            tma_load_page(dst + p * C::PART_BYTES + ((lane >> 3) * PA_TILE + ((lane & 7) << box_log)) * 128, map, p * 64, slot & ((1 << a.pg.page_log) - 1), h, page, bar);
        }
        __syncwarp();
      };
      if (i >= ST) wait(kempty + 8 * stage, use - 1);
      // (warps without rows in this unit have no part in its products: nothing else holds the ring back for them)
      if (i >= 4) wait(taken + 8 * (i & 3), (i >> 2) - 1);
      if (!ok) break;
      if (lane == 0) {
        sh.valid[i & 3][0] = v[0] | (unsigned long long)v[1] << 32;
        sh.valid[i & 3][1] = v[2] | (unsigned long long)v[3] << 32;
        mbar_arrive(info + 8 * (i & 3));
      }
      issue(keys0 + stage * C::TILE_BYTES, &mapK, kfull + 8 * stage, i >= a.miss_from ? 16 : 0);
      keys = i + 1;
      if (first) {
        if (i) wait(kempty + 8 * ((i - 1) % ST), (i - 1) / ST);          // the queries' last products are done
        if (!ok) break;
        const int row0 = at.u / Hkv * ROWS, halves = at.halves<QT>(a, span);
        if (q_tma) {
          if (lane == 0) mbar_expect_tx(q_ready, halves * C::TILE_BYTES);
          __syncwarp();
          if (lane < halves * PARTS) {
            const int q = lane / PARTS, p = lane % PARTS;
            tma_load_queries(smem0 + q * C::TILE_BYTES + p * C::PART_BYTES, &mapQ, p * 64, h * a.group, at.b * a.M + token_of(a, row0 + q * 128), q_ready);
          }
        } else {
          constexpr int CPR = C::RB / 16;          // 16-byte chunks of a row
#pragma unroll 4
          for (int e = lane; e < halves * 128 * CPR; e += 32) {
            const int r = e / CPR, chunk = e % CPR;
            const bool in = row0 + r < R;
            const int tok = in ? token_of(a, row0 + r) : 0, head = h * a.group + (in ? row0 + r - tok * a.group : 0);
            const char *src = reinterpret_cast<const char *>(a.q) + (((long long)at.b * a.M + tok) * a.q_stride + (long long)head * D) * 2 + chunk * 16;
            const uint32_t dst = smem0 + r / 128 * C::TILE_BYTES + chunk / 8 * C::PART_BYTES + r % 128 * 128 + ((chunk & 7) ^ (r & 7)) * 16;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
          }
          asm volatile("cp.async.wait_all;" ::: "memory");
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(q_ready);
        }
        ++queries;
      }
      if (i >= ST) wait(vempty + 8 * stage, use - 1);
      if (!ok) break;
      issue(values0 + stage * C::TILE_BYTES, &mapV, vfull + 8 * stage, 0);
      values = i + 1;
    }
  } else if (warp == C::WARPS + 1) {
    // ---------------- products (the warp as a whole, one lane issues)
    constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);
    constexpr uint32_t idesc_o = idesc | (1u << 16) | ((64u >> 3) << 17);
    TreeWalk at(a, run, ROWS);
    int units = 0, turns[2] = {0, 0};
    // S of rows 128 q .. of tile i
    auto scores = [&](int i, int q, int halves) {
      const int stage = i % ST;
      if (q == 0) {
        if (i == 0 || at.t == 0) wait(q_ready, units++);
        wait(kfull + 8 * stage, i / ST);
      }
      if (!ok) return;
      tc_fence_after();
      if (leader) {
        const bool two = at.two();
        const uint64_t dq = umma_smem_desc(smem0 + q * C::TILE_BYTES), dk = umma_smem_desc(keys0 + stage * C::TILE_BYTES);
        const uint32_t idesc_s = idesc | ((two ? 128u : 64u) >> 3) << 17;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t off = (uint64_t)(k / 4 * (C::PART_BYTES >> 4) + k % 4 * 2);
          umma_bf16(tmem + 128 * q, dq + off, dk + off, idesc_s, k ? 1u : 0u);
        }
        if (q + 1 == halves) umma_commit(kempty + 8 * stage);
        umma_commit(s_full + 8 * q);
      }
      __syncwarp();
    };
    int halves = at.halves<QT>(a, at.span(a, ROWS));
    for (int q = 0; q < halves; ++q) scores(0, q, halves);
    for (int i = 0; i < run.count && ok; ++i) {
      const int stage = i % ST, now = halves;
      const bool first = i == 0 || at.t == 0, two = at.two(), more = i + 1 < run.count;
      if (more) {
        at.next(a, ROWS);
        if (QT == 2 && at.t == 0) halves = at.halves<QT>(a, at.span(a, ROWS));
      }
      for (int q = 0; q < QT && ok; ++q) {
        if (q < now) {
          wait(p_ready + 8 * q, turns[q]++);
          if (q == 0) wait(vfull + 8 * stage, i / ST);
          if (!ok) break;
          tc_fence_after();
          if (leader) {
            const uint64_t dv = umma_smem_desc(values0 + stage * C::TILE_BYTES);
#pragma unroll
            for (int k = 0; k < 8; ++k) {          // 16 slots: two groups of eight rows, 2 KB
              if (k >= 4 && !two) break;
#pragma unroll
              for (int p = 0; p < PARTS; ++p)
#pragma unroll
                for (int low = 0; low < 2; ++low)
                  umma_bf16_ts(tmem + C::O + D * q + 64 * p, tmem + 128 * q + 16 * k + 8 * low, dv + (uint64_t)(p * (C::PART_BYTES >> 4) + 128 * k), idesc_o,
                               first && k == 0 && !low ? 0u : 1u);
            }
            if (q + 1 == now) umma_commit(vempty + 8 * stage);
            umma_commit(o_full + 8 * q);
          }
          __syncwarp();
        }
        if (more && q < halves) scores(i + 1, q, halves);
      }
    }
  } else {
    // ---------------- softmax
    const int q = warp >> 3, w4 = warp & 3, part = warp >> 2 & 1, row = w4 * 32 + lane, meeting = 1 + q * 4 + w4;
    const uint32_t trow = tmem + ((uint32_t)(w4 * 32) << 16), mine = trow + 128 * q + part * 64, sums = trow + C::O + D * q + part * (D / 2);
    const float scale = a.scale2 == 0.f ? 1.f : fabsf(a.scale2);
    const uint64_t scale2 = f32x2(scale, scale);
    TreeWalk at(a, run, ROWS);
    int2 open = make_int2(0, 0);
    int looks = 0, turn = 0;                       // turn: tiles of this warp's rows
    bool from_start = false, idle = false, seen = false;       // seen: a tile held something that the row sees
    unsigned long long spoiled = 0;                // this thread's columns in which the row sees a value that is not finite
    auto row_of = [&]() { return at.u / Hkv * ROWS + q * 128 + row; };
    float m = TREE_TC_SLACK, l = 0.f;              // the reference; the sum of this thread's slots
    for (int i = 0; i < run.count; ++i, at.next(a, ROWS)) {
      const int stage = i % ST, use = i / ST;
      const bool first = i == 0 || at.t == 0;
      if (first) {
        const PagedSpan span = at.span(a, ROWS);
        const int row0 = at.u / Hkv * ROWS;
        from_start = at.t == 0;
        idle = q >= at.halves<QT>(a, span);
        open = paged_tree_open(a, span, token_of(a, row0), min(span.n_new, token_of(a, min(R, row0 + ROWS) - 1) + 1) - 1);
        m = TREE_TC_SLACK, l = 0.f, seen = false, spoiled = 0;
      }
      const bool two = at.two(), here = part == 0 || two;
      const int base0 = at.base(0), base1 = at.base(1);
      wait(info + 8 * (i & 3), i >> 2);
      const unsigned long long valid0 = sh.valid[i & 3][0], valid1 = sh.valid[i & 3][1];
      __syncwarp();
      if (lane == 0) mbar_arrive(taken + 8 * (i & 3));
      const bool open0 = valid0 == ~0ull && base0 >= open.x && base0 + PA_TILE <= open.y, open1 = !two || (valid1 == ~0ull && base1 >= open.x && base1 + PA_TILE <= open.y);
      const bool all = part ? open1 : open0;       // every row sees every slot of this block
      if (idle) {
        looks += !(open0 && open1);
        continue;
      }
      wait(s_full + 8 * q, turn);
      unsigned long long sees = ~0ull;             // slots of the block that this row sees
      if (!all) {
        const PagedSpan span = at.span(a, ROWS);
        const int token = row_of() < R ? token_of(a, row_of()) : a.M;
        sees = here ? (part ? valid1 : valid0) & paged_tree_bits(a, span, paged_tree_range(a, span, at.b, token), at.b, token, part ? base1 : base0) : 0ull;
      }
      tc_fence_after();
      // The reference may move behind any 16 slots; where it did, the tile's probabilities are brought to the last one when they are all there: products
      // with powers of two, exact in both parts.
      float ref = m, refs[4];
      bool any = seen, moved = false;              // the row saw something by here; its reference moved in this tile
      uint64_t sum = 0;
      if (here) {
        float s[2][16];                            // 16 slots; the next ones are on their way meanwhile
        tmem_load16(mine, s[0]);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          float(&y)[16] = s[x & 1];
          tmem_wait16(y);
          if (x < 3) tmem_load16(mine + 16 * (x + 1), s[(x + 1) & 1]);
          if (a.scale2 <= 0.f) {
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = a.scale2 < 0.f ? -y[e] : y[e] * 0.f;
          }
          if (!all) {
            const uint32_t bits = (uint32_t)(sees >> 16 * x);
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = bits >> e & 1 ? y[e] : -INFINITY;
          }
          float t[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int e = 0; e < 16; e += 2) asm("max.f32 %0, %0, %1, %2;" : "+f"(t[e >> 1 & 1]) : "f"(y[e]), "f"(y[e + 1]));
          const float top = fmaxf(t[0], t[1]) * scale;
          if (top > ref || (!any && top < ref - 2 * TREE_TC_SLACK && top > -INFINITY)) {
            const float now = ceilf(top) + TREE_TC_SLACK, f = any ? flash_ex2(ref - now) : 0.f;
            sum = mul2(sum, f32x2(f, f));
            ref = now;
            moved = true;
          }
          any |= top > -INFINITY;
          refs[x] = ref;
          const uint64_t minus = f32x2(-ref, -ref);
          uint64_t here2 = 0;
          uint32_t p[16];                          // high parts, low parts
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 d = unpack2(fma2(f32x2(y[2 * e], y[2 * e + 1]), scale2, minus));
            const float p0 = flash_ex2(d.x), p1 = flash_ex2(d.y);
            here2 = add2(here2, f32x2(p0, p1));
            p[e] = pack_bf16x2(p0, p1);
            const float2 low = unpack2(fma2(f32x2(__uint_as_float(p[e] << 16), __uint_as_float(p[e] & 0xffff0000u)), f32x2(-1.f, -1.f), f32x2(p0, p1)));
            p[8 + e] = pack_bf16x2(low.x, low.y);
          }
          sum = add2(sum, here2);
          tmem_st16(mine + 16 * x, p);
        }
      }
      const float2 both = unpack2(sum);
      float mass = both.x + both.y;
      const float own = any ? ref : -INFINITY;
      sh.top[q][part][row] = own;
      const bool again = bar_any64(meeting, moved);
      const float other = sh.top[q][part ^ 1][row];        // (written again only after this warp's next probabilities)
      if (again) {                                 // (both warps of these rows)
        const float now = fmaxf(own, other);       // (-inf: nothing seen as yet)
        const float alpha = seen ? flash_ex2(m - now) : 1.f;
        // (slots before the first one that the row sees have probabilities 0 and may have a larger reference)
        auto factor = [&](float r) { return flash_ex2(fminf(r - now, 0.f)); };
        if (here) {
          tmem_stored();
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const __nv_bfloat162 f = __float2bfloat162_rn(factor(refs[x]));
            float y[16];
            tmem_load16(mine + 16 * x, y);
            tmem_wait16(y);
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const __nv_bfloat162 z = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&y[e]), f);
              w[e] = *reinterpret_cast<const uint32_t *>(&z);
            }
            tmem_st16(mine + 16 * x, w);
          }
        }
        mass *= factor(ref);
        l *= alpha;
        if (now > -INFINITY) m = now;
        if (!first && __any_sync(0xffffffffu, alpha != 1.f)) {
          wait(o_full + 8 * q, turn - 1);
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D / 2; c += 16) {
            float o[16];
            tmem_load16(sums + c, o);
            tmem_wait16(o);
            uint32_t r[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(o[e] * alpha);
            tmem_st16(sums + c, r);
          }
        }
      }
      seen = any || other > -INFINITY;
      if (here) l += mass;
      if (!(open0 && open1)) {
        // The two threads of a row of the first 128 look at slot `row` of the tile; all warps wait for theirs, like all roles with a limit.  (The
        // second 128 rows' products follow the first's.)
        uint4 *v = reinterpret_cast<uint4 *>(smem + (values0 - smem0) + stage * C::TILE_BYTES + (PARTS == 2 ? part * C::PART_BYTES : 0) + row * 128);
        constexpr int CH = PARTS == 2 ? 8 : 4;     // 16-byte chunks of a thread: its half of the columns
        auto chunk = [&](int x) -> uint4 & { return v[((PARTS == 2 ? x : part * 4 + x) ^ row) & 7]; };
        uint32_t *const found = sh.bad[looks & 3][part];
        if (q == 0) {
          wait(vfull + 8 * stage, use);
          if (!((row < 64 ? valid0 : valid1) >> (row & 63) & 1)) {
#pragma unroll
            for (int x = 0; x < CH; ++x) chunk(x) = make_uint4(0u, 0u, 0u, 0u);
          } else if (!(row < 64 ? open0 : open1)) {
            auto ones = [](uint32_t w) { return (w & 0x7f807f80u) + 0x00800080u; };      // (an exponent of all ones carries into its sign)
            uint32_t bad = 0;
#pragma unroll
            for (int x = 0; x < CH; ++x) {
              const uint4 w = chunk(x);
              bad |= ones(w.x) | ones(w.y) | ones(w.z) | ones(w.w);
            }
            if (bad & 0x80008000u) {
              unsigned long long gone = 0;
#pragma unroll 1
              for (int x = 0; x < CH; ++x)
#pragma unroll 1
                for (int e = 0; e < 4; ++e) {
                  uint32_t &w = (&chunk(x).x)[e];
                  const uint32_t y = ones(w);
                  gone |= (unsigned long long)((y >> 15 & 1) | (y >> 30 & 2)) << (8 * x + 2 * e);
                  w &= (y & 0x8000u ? 0u : 0xffffu) | (y >> 31 ? 0u : 0xffff0000u);
                }
              sh.columns[looks & 1][row][part] = gone;
              atomicOr(found + (row >> 5), 1u << (row & 31));
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(looked + 8 * (looks & 1));
        }
        wait(looked + 8 * (looks & 1), looks >> 1);
        if (found[0] | found[1] | found[2] | found[3]) {
          const PagedSpan span = at.span(a, ROWS);
          const int token = row_of() < R ? token_of(a, row_of()) : a.M;
          const int2 range = paged_tree_range(a, span, at.b, token);
#pragma unroll 1
          for (int x = 0; x < 2; ++x) {
            unsigned long long bits = (found[2 * x] | (unsigned long long)found[2 * x + 1] << 32) & (x ? valid1 : valid0);
            bits &= bits ? paged_tree_bits(a, span, range, at.b, token, x ? base1 : base0) : 0ull;
            for (; bits; bits &= bits - 1) spoiled |= sh.columns[looks & 1][64 * x + __ffsll(bits) - 1][part];
          }
        }
        // (the one after next: who comes last is one tile behind)
        if (q == 0 && tid < 8) (&sh.bad[(looks + 2) & 3][0][0])[tid] = 0;
        ++looks;
      }
      tmem_stored();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_ready + 8 * q);

      if (at.t + 1 == at.tiles() || i + 1 == run.count) {
        // the unit, or this CTA's part of it, ends
        sh.sum[q][part][row] = l;
        bar_any64(meeting, false);
        l = sh.sum[q][0][row] + sh.sum[q][1][row];
        wait(o_full + 8 * q, turn);
        // (a warp whose own waits were met has its rows' product from what the others left: all of them say so before the product starts)
        if (!ok || sh.dead) l = NAN;
        tc_fence_after();
        const int r = row_of(), h = at.u % Hkv;
        const bool whole = from_start && at.t + 1 == at.tiles(), live = r < R && token_of(a, r) < at.span(a, ROWS).n_new;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const long long part_row = (long long)(2 * blockIdx.x + from_start) * ROWS + q * 128 + row;
        float *dst_o = a.part_o + part_row * D + part * (D / 2);
        bf16 *dst = live ? paged_out_row<bf16>(a, at.b, h, r, D) + part * (D / 2) : nullptr;
#pragma unroll 1
        for (int c = 0; c < D / 2; c += 16) {
          float o[16];
          tmem_load16(sums + c, o);
          tmem_wait16(o);
          if (spoiled >> c & 0xffff) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (spoiled >> (c + e) & 1) o[e] = l == 0.f ? 0.f : NAN;
          }
          if (whole) {
            if (live) {
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(o[8 * x + 2 * e] * inv, o[8 * x + 2 * e + 1] * inv);
                *reinterpret_cast<uint4 *>(dst + c + 8 * x) = make_uint4(w[0], w[1], w[2], w[3]);
              }
            }
          } else if (r < R) {
#pragma unroll
            for (int x = 0; x < 4; ++x) *reinterpret_cast<float4 *>(dst_o + c + 4 * x) = make_float4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
          }
        }
        if (part == 0 && whole && live) paged_write_lse(a, at.b, h, r, m, l);
        if (part == 0 && !whole && r < R) a.part_ml[part_row] = make_float2(l == 0.f ? -INFINITY : m, l);
        tc_fence_before();                         // (the next unit's products wait for this warp's next probabilities)
      }
      ++turn;
    }
  }
  tc_fence_before();
  // Nothing that was asked for may outlive the CTA.  Where every wait was met all of it has been waited for; where one ran out, in whichever warp, copies
  // and products get another limit each.
  const bool late = __syncthreads_or(!ok);
  if (warp == C::WARPS) {
    if (late) {
      for (int i = max(0, keys - ST); i < keys; ++i) tile_arrived(kfull + 8 * (i % ST), (i / ST) & 1, a.wait_ns);
      for (int i = max(0, values - ST); i < values; ++i) tile_arrived(vfull + 8 * (i % ST), (i / ST) & 1, a.wait_ns);
      if (queries) tile_arrived(q_ready, (queries - 1) & 1, a.wait_ns);
    }
  } else if (warp == C::WARPS + 1) {
    if (late) {
      if (leader) umma_commit(drained);
      __syncwarp();
      tile_arrived(drained, 0, a.wait_ns);
    }
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)C::COLS) : "memory");
  }
}

}  // namespace tsfm
