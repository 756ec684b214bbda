"""Serving over a cache of pages on the GPU, at the edges of what a call may be given: values that are not finite in the slots or queries
of some tokens only."""
import math

import pytest
import torch

from tests.serving_ref import Pool
from tests.test_gpu_serving import BF16, F32, check_attention, ints, lib, stream, wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("bad", ["query", "nan key", "inf key", "old key"])
def test_weights_of_slots_that_a_bad_row_does_not_see(dtype, window, bad):
    """A NaN query, or a key that some tokens see and others do not: out and lse of the rows that do not see it, and the weights of the slots
    that no row with it sees, are bit for bit those of the call without it; the others are not finite."""
    tsfm = lib()
    B, M, Hq, Hkv, D, n = 2, 5, 4, 2, 64, 150
    pool = Pool(B, Hkv, D, 16, [n + M] * B, dtype, seed=4)
    q = wide((B, M), Hq * D, dtype, 0, 5)
    w_in = torch.rand(B, Hkv, n + M, generator=torch.Generator().manual_seed(6)).cuda()
    pages = pool.describe(tsfm)
    work = torch.empty(tsfm.tsfm_paged_attention_workspace(pages, B, M, Hq, n + M, True), dtype=torch.uint8, device="cuda")
    slot = n - 39 if bad == "old key" else n + 2
    got = []
    for spoilt in (False, True):
        if spoilt and bad == "query":
            q[0, 2, :D] = math.nan                             # token 2, head 0: key head 0
        elif spoilt:
            pool.put(pool.k, 0, slot, math.inf if bad == "inf key" else math.nan)
        out, lse, w = torch.zeros(B, M, Hq * D, dtype=dtype, device="cuda"), torch.zeros(B, M, Hq, device="cuda"), torch.zeros_like(w_in)
        tsfm.tsfm_paged_attention(stream(), pages, q, q.stride(1), out, out.stride(1), ints([n] * B), None, B, M, Hq, 0.1, True, window, n + M, lse, w_in, w,
                                  n + M, work, work.numel())
        got.append((out.cpu().view(B, M, Hq, D), lse.cpu(), w.cpu()))
    (out0, lse0, w0), (out1, lse1, w1) = got
    spoilt_row = torch.zeros(B, M, Hq, dtype=torch.bool)
    spoilt_slot = torch.zeros(B, Hkv, n + M, dtype=torch.bool)
    for m in range(M):
        start, end = max(0, n + m + 1 - window) if window else 0, n + m + 1
        for h in range(Hq):
            if (m == 2 and h == 0) if bad == "query" else start <= slot < end:
                spoilt_row[0, m, h] = True
                spoilt_slot[0, h * Hkv // Hq, start:end] = True
    assert spoilt_row.any() and not spoilt_slot.all()
    assert torch.equal(out0[~spoilt_row], out1[~spoilt_row]) and torch.equal(lse0[~spoilt_row], lse1[~spoilt_row])
    assert not torch.isfinite(out1[spoilt_row]).any() and not torch.isfinite(lse1[spoilt_row]).any()
    assert torch.equal(w0[~spoilt_slot], w1[~spoilt_slot]) and torch.isfinite(w0).all()
    assert not torch.isfinite(w1[spoilt_slot]).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_bad_row_gives_nothing_to_slots_of_pages_outside_the_pool(dtype):
    tsfm = lib()
    Hq, Hkv, D, n = 2, 1, 64, 100
    pool = Pool(1, Hkv, D, 16, [n], dtype, seed=4)
    pool.table[0, 3] = pool.k.shape[0]                         # slots 48 to 63
    q = torch.full((1, 1, Hq * D), math.nan, dtype=dtype, device="cuda")
    pages = pool.describe(tsfm)
    work = torch.empty(tsfm.tsfm_paged_attention_workspace(pages, 1, 1, Hq, n, True), dtype=torch.uint8, device="cuda")
    out, w = torch.zeros_like(q), torch.ones(1, Hkv, n, device="cuda")
    tsfm.tsfm_paged_attention(stream(), pages, q, Hq * D, out, Hq * D, ints([n]), None, 1, 1, Hq, 0.1, False, 90, n, None, w, w, n, work, work.numel())
    assert int(pool.status) == tsfm.TSFM_PAGES_BAD_ID
    hidden = torch.zeros(n, dtype=torch.bool)
    hidden[:10], hidden[48:64] = True, True                    # before the window; in no page
    assert (w[0, 0].cpu()[hidden] == 1).all() and w[0, 0].cpu()[~hidden].isnan().all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,Hq,Hkv,M,page,lengths", [(64, 4, 2, 1, 16, [40] * 1000), (128, 16, 2, 2, 64, [2000, 1, 300]), (32, 20, 1, 2, 8, [500] * 3)])
@pytest.mark.parametrize("miss_from", [0, 1])
def test_a_tile_that_does_not_arrive(dtype, D, Hq, Hkv, M, page, lengths, miss_from):
    """All copies land, but a CTA waits for 16 bytes more from its first or second tile on: the wait ends, the call reports it, what depends on the
    tile is NaN and the rest is right.  The next call, without it, is as before."""
    tsfm = lib()
    B, n = len(lengths), max(lengths) + M
    pool = Pool(B, Hkv, D, page, [x + M for x in lengths], dtype, seed=3)
    pages, q = pool.describe(tsfm), wide((B, M), Hq * D, dtype, 0, 8)
    work = torch.empty(tsfm.tsfm_paged_attention_workspace(pages, B, M, Hq, n, True), dtype=torch.uint8, device="cuda")

    def attend():
        out, lse = torch.zeros(B, M, Hq * D, dtype=dtype, device="cuda"), torch.zeros(B, M, Hq, device="cuda")
        w = torch.full((B, Hkv, n), -9.0, device="cuda")
        tsfm.tsfm_paged_attention(stream(), pages, q, Hq * D, out, Hq * D, ints(lengths), None, B, M, Hq, 0.1, True, 0, n, lse, None, w, n, work, work.numel())
        torch.cuda.synchronize()
        status = int(pool.status)
        pool.status.zero_()
        return out.cpu().view(B, M, Hq, D), lse.cpu(), w.cpu(), status
    good = attend()
    assert good[3] == 0
    tsfm.tsfm_debug_tile_wait(2000, miss_from)
    try:
        bad = attend()
    finally:
        tsfm.tsfm_debug_tile_wait()
    lost = bad[1].isnan()
    assert torch.equal(bad[0].isnan().all(-1), lost) and torch.equal(bad[0].isnan().any(-1), lost)
    assert torch.equal(bad[0][~lost], good[0][~lost]) and torch.equal(bad[1][~lost], good[1][~lost])
    if miss_from == 0:
        assert bad[3] == tsfm.TSFM_PAGES_TIMEOUT and lost.all()
        seen = torch.arange(n) < torch.tensor(lengths)[:, None, None] + M
        assert bad[2][seen.expand_as(bad[2])].isnan().all() and (bad[2][~seen.expand_as(bad[2])] == -9).all()
    elif B == 1000:                                            # four units a CTA, the first one whole
        assert bad[3] == tsfm.TSFM_PAGES_TIMEOUT and lost.any() and not lost.all()
    again = attend()
    assert again[3] == 0 and all(torch.equal(x, y) for x, y in zip(again[:3], good[:3]))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("window", [0, 128, 3])
@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 64), (3, 1, 128)])
def test_prompts_beside_single_tokens(dtype, window, Hq, Hkv, D):
    """Hundreds of new tokens, from an empty cache and behind a long one, beside series that bring one token or none: units whose rows do not exist,
    rows that see a small part of what their unit reads."""
    M, lengths, new = 300, [0, 500, 63, 1000, 7], [300, 1, 131, 0, 300]
    pool = Pool(len(lengths), Hkv, D, 16, [n + m for n, m in zip(lengths, new)], dtype, seed=D)
    check_attention(pool, dtype, Hq, Hkv, D, lengths, new, M, True, window, weights=True, qpad=8)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_captured_attention_and_eviction_on_another_stream(dtype):
    """Both from one graph, replayed with other queries and lengths, against calls of their own; series longer than the capture saw, and shorter ones."""
    tsfm = lib()
    B, Hq, Hkv, D, page, longest, budget = 3, 8, 2, 64, 16, 5000, 300
    pool = Pool(B, Hkv, D, page, [longest] * B, dtype, seed=9, spare=B * -(-budget // page))
    dst = ints([pool.spare_ids[b::B] for b in range(B)])
    pages, side = pool.describe(tsfm), torch.cuda.Stream()
    size = tsfm.tsfm_paged_attention_workspace(pages, B, 1, Hq, longest, True)
    work = torch.empty(size, dtype=torch.uint8, device="cuda")
    q, length = torch.zeros(B, 1, Hq * D, dtype=dtype, device="cuda"), ints([1] * B)
    names = dict(out=torch.zeros_like(q), w=torch.zeros(B, Hkv, longest, device="cuda"), w_out=torch.zeros(B, Hkv, budget, device="cuda"),
                 kept=torch.zeros(B, Hkv, budget, dtype=torch.int32, device="cuda"), len_out=torch.zeros_like(length))

    def both(s):
        tsfm.tsfm_paged_attention(s, pages, q, Hq * D, names["out"], Hq * D, length, None, B, 1, Hq, 0.125, False, 0, longest, None, None, names["w"], longest, work, size)
        tsfm.tsfm_cache_evict(s, pages, dst, dst.shape[1], length, names["w"], longest, B, budget, 4, 50, longest, names["kept"], names["w_out"], budget, names["len_out"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both(torch.cuda.current_stream().cuda_stream)
    k0 = pool.k.clone()
    for i, lengths in enumerate(([4000, 10, 0], [5000, 301, 300], [1, 4097, 2500])):
        q.copy_(wide((B, 1), Hq * D, dtype, 0, 30 + i))
        length.copy_(ints(lengths))
        got = []
        for replay in (True, False):
            pool.k.copy_(k0)
            for t in names.values():
                t.fill_(7)
            torch.cuda.synchronize()
            if replay:
                with torch.cuda.stream(side):
                    graph.replay()
            else:
                both(stream())
            torch.cuda.synchronize()
            got.append([t.clone() for t in (*names.values(), pool.k)])
        assert all(torch.equal(x, y) for x, y in zip(*got))
        assert got[0][4].tolist() == [min(n, budget) for n in lengths] and int(pool.status) == 0
