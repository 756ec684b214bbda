"""Serving over a cache of pages on the GPU against the definitions in 64 bits (tests/serving_ref.py)."""
import math

import numpy as np
import pytest
import torch

from oracle import tsfm_oracle as orc
from tests import serving_ref as ref
from tests.serving_ref import U, Pool

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def lib():
    import paper_2511_18191_b200 as tsfm
    return tsfm


def stream():
    return torch.cuda.current_stream().cuda_stream


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def wide(rows, width, dtype, pad, seed, factor=1.0):
    """[*rows, width] of normals inside rows that are `pad` elements longer, NaN in the padding."""
    g = torch.Generator().manual_seed(seed)
    x = torch.full((*rows, width + pad), math.nan)
    x[..., :width] = torch.randn((*rows, width), generator=g) * factor
    return x.to(dtype).cuda()[..., :width]


# ------------------------------------------------------------------------------------------ rotary positions and append
ROPES = [("half", 64, "plain", 64), ("half", 32, "linear", 64), ("half", 128, "parts", 128), ("interleaved", 64, "base", 64),
         ("interleaved", 32, "parts", 128), ("half", 16, "plain", 32), ("half", 24, "linear", 64), ("half", 2, "plain", 32), ("half", 6, "parts", 128),
         ("interleaved", 2, "plain", 32), ("interleaved", 30, "base", 32), ("half", 0, "plain", 64), ("interleaved", 0, "plain", 64)]
SCALING = {"plain": 0, "linear": 1, "base": 2, "parts": 3}


def make_rope(layout, rot, scaling, mscale=1.0):
    args = (1e4, 8.0, 4096.0, 1.0, 32.0)
    f = ref.frequencies(rot, args[0], scaling, *args[1:])
    return lib().tsfm_rope_init(0 if layout == "half" else 1, rot, SCALING[scaling], *args, mscale), f


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout,rot,scaling,D", ROPES)
@pytest.mark.parametrize("B,M,Hq,Hkv,page,order,inplace,pad", [
    (1, 1, 4, 4, 16, "heads", False, 0), (5, 9, 10, 2, 8, "slots", True, 16), (3, 70, 3, 1, 64, "heads", False, 8)])
def test_rope_append(dtype, layout, rot, scaling, D, B, M, Hq, Hkv, page, order, inplace, pad):
    tsfm = lib()
    rng = np.random.default_rng(rot + D + B)
    length = rng.integers(0, 100, B)
    new = [M] + [int(x) for x in rng.integers(0, M + 1, B - 1)]
    pos = [int(x) for x in rng.integers(0, 2 ** 21, B)]
    pos[-1] = 2 ** 31 - 1 - M                                  # as far as positions go
    pool = Pool(B, Hkv, D, page, length + M, dtype, order, seed=B, fill=7.0)
    qkv = wide((B, M), (Hq + 2 * Hkv) * D, dtype, pad, seed=D)
    before = qkv.cpu().double()
    q_out = qkv if inplace else torch.full((B, M, Hq * D), -3.0, dtype=dtype, device="cuda")
    rope, f = make_rope(layout, rot, scaling, 1.25)
    tsfm.tsfm_rope_append(stream(), rope, pool.describe(tsfm), qkv, qkv.stride(1), q_out, q_out.stride(1), ints(pos), ints(length), ints(new), B, M, Hq)
    torch.cuda.synchronize()
    # one rounding of the result; in 32 bits each of the two products, their sum, cos and sin (two steps each, mscale) and the
    # angle (2^-25 turns of the float, 2 pi 2^-25 < 2^-22); the reference's own angle pos * f (f to two steps, the product) in 64
    tol = lambda x, want, at: U[dtype] * want.abs() + (2.0 ** -22 + 8 * 2.0 ** -24 + at * 2.0 ** -51) * 1.25 * 2 * x.abs().max()
    got_q, gk, gv = q_out.cpu().double()[..., :Hq * D], pool.k.cpu(), pool.v.cpu()
    touched = torch.zeros(gk.shape[0], page, dtype=torch.bool)
    for b in range(B):
        for m in range(M):
            x = before[b, m].view(Hq + 2 * Hkv, D)
            if m >= new[b]:
                assert torch.equal(got_q[b, m], before[b, m, :Hq * D] if inplace else torch.full((Hq * D,), -3.0, dtype=torch.float64))
                continue
            want = ref.turn(x[:Hq + Hkv], float(pos[b] + m), f, layout, 1.25)
            assert ((got_q[b, m].view(Hq, D) - want[:Hq]).abs() <= tol(x, want[:Hq], pos[b] + m)).all()
            slot = int(length[b]) + m
            page_id = int(pool.table[b, slot // page])
            touched[page_id, slot % page] = True
            assert ((gk[page_id, :, slot % page].double() - want[Hq:]).abs() <= tol(x, want[Hq:], pos[b] + m)).all()
            assert torch.equal(gv[page_id, :, slot % page].double(), x[Hq + Hkv:])
            # what does not turn is copied
            assert torch.equal(gk[page_id, :, slot % page, rot:].double(), x[Hq:Hq + Hkv, rot:])
    rest = ~touched[:, None, :, None].expand(gk.shape)
    assert (gk[rest] == 7).all() and (gv[rest] == 7).all() and int(pool.status) == 0
    if inplace:                                                # keys and values of the input stay
        assert torch.equal(qkv.cpu().double()[..., Hq * D:], before[..., Hq * D:])


def test_rope_append_without_queries_positions_and_counts():
    """q_out NULL, pos NULL (slot numbers), n_new NULL (all): as a draft's cache that catches up; and n_heads 0."""
    tsfm = lib()
    B, M, Hkv, D = 2, 5, 2, 64
    for Hq in (6, 0):
        pool = Pool(B, Hkv, D, 16, [20, 40], F32, fill=0.0)
        qkv = wide((B, M), (Hq + 2 * Hkv) * D, F32, 0, 1)
        rope, f = make_rope("half", D, "plain")
        tsfm.tsfm_rope_append(stream(), rope, pool.describe(tsfm), qkv, qkv.stride(1), None, 0, None, ints([15, 30]), None, B, M, Hq)
        for b, n in enumerate([15, 30]):
            k = pool.rows(pool.k, b, n + M)
            for m in range(M):
                x = qkv[b, m].cpu().double().view(-1, D)[Hq:Hq + Hkv]
                assert (k[n + m] - ref.turn(x, float(n + m), f, "half")).abs().max() <= 2.0 ** -20 * x.abs().max()


def test_appends_outside_the_pool_are_dropped_and_reported():
    tsfm = lib()
    B, M, Hkv, D, page = 5, 4, 2, 32, 8
    for layout, rot in (("half", 32), ("half", 6)):
        pool = Pool(B, Hkv, D, page, [16] * B, BF16, fill=5.0, spare=2)
        pool.table[1, 1] = pool.k.shape[0]                     # one past the pool
        pool.table[2, 0] = -7
        length = ints([0, 6, 7, 14, -3])                       # b = 3 runs over its 16 slots, b = 4 is below 0
        qkv = wide((B, M), (2 + 2 * Hkv) * D, BF16, 0, 3)
        q_out = torch.zeros(B, M, 2 * D, dtype=BF16, device="cuda")
        rope, _ = make_rope(layout, rot, "plain")
        tsfm.tsfm_rope_append(stream(), rope, pool.describe(tsfm), qkv, qkv.stride(1), q_out, q_out.stride(1), None, length, None, B, M, 2)
        torch.cuda.synchronize()
        assert int(pool.status) == tsfm.TSFM_PAGES_BAD_ID | tsfm.TSFM_PAGES_BAD_LEN
        v = pool.v.cpu()
        written = (v != 5).any(3).any(1)                       # [page, slot]
        want = torch.zeros_like(written)
        t = pool.table.cpu()
        for b, slots in enumerate([[0, 1, 2, 3], [6, 7], [8, 9, 10], [14, 15], [0]]):
            for s in slots:
                want[t[b, s // page], s % page] = True
        assert torch.equal(written, want)
        assert (q_out.abs().sum(2) > 0).all()                  # the queries are turned all the same


# ------------------------------------------------------------------------------------------ attention
def check_attention(pool, dtype, Hq, Hkv, D, length, new, M, causal=True, window=0, weights=False, max_len=None, qpad=0, scale=None, w_null=False,
                    seed=0, qfactor=2.0, expect_status=0):
    tsfm = lib()
    B = pool.B
    total = [n + (m if causal else 0) for n, m in zip(length, new)]
    max_len = max_len or max(1, max(total))
    scale = scale if scale is not None else 1 / math.sqrt(D)
    q = wide((B, M), Hq * D, dtype, qpad, seed + 1, qfactor)
    out_wide = torch.full((B, M, Hq * D + qpad), -9.0, dtype=dtype, device="cuda")
    lse = torch.full((B, M, Hq), -9.0, device="cuda")
    w_in = torch.rand(B, Hkv, max_len + 3, generator=torch.Generator().manual_seed(seed)).cuda() if weights else None
    w_out = torch.full_like(w_in, -9.0) if weights else None
    pages = pool.describe(tsfm)
    size = tsfm.tsfm_paged_attention_workspace(pages, B, M, Hq, max_len, weights)
    work = torch.full((size + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    tsfm.tsfm_paged_attention(stream(), pages, q, q.stride(1), out_wide, out_wide.stride(1), ints(length), ints(new), B, M, Hq, scale, causal, window,
                              max_len, lse, None if w_null else w_in, w_out, max_len + 3, work, size)
    torch.cuda.synchronize()
    assert int(pool.status) == expect_status
    assert (work[size:] == 0xA5).all()
    got, glse, gw = out_wide.cpu().double(), lse.cpu().double(), w_out.cpu().double() if weights else None
    assert (got[..., Hq * D:] == -9).all()
    for b in range(B):
        k, v = pool.rows(pool.k, b, total[b]), pool.rows(pool.v, b, total[b])
        seen = torch.zeros(Hkv, total[b], dtype=torch.float64)
        wtol = torch.zeros(Hkv, total[b], dtype=torch.float64)
        for m in range(M):
            if m >= new[b]:
                assert (got[b, m, :Hq * D] == -9).all() and (glse[b, m] == -9).all()
                continue
            end = min(length[b] + m + 1 if causal else length[b], total[b])
            start = max(0, end - window) if window else 0
            o, z, p, absv, peak = ref.attention(q[b, m].cpu().double().view(Hq, D), k, v, scale, start, end)
            rel = ref.attention_tolerance(dtype, D, end - start, peak)[:, None]
            err = (got[b, m, :Hq * D].view(Hq, D) - o).abs()
            assert (err <= U[dtype] * o.abs() + rel * absv + 1e-30).all(), (b, m, float(err.max()))
            if end > start:
                assert ((glse[b, m] - z).abs() <= rel[:, 0] + 4 * U[F32] * (z.abs() + peak + 1)).all(), (b, m)
            else:
                assert (glse[b, m] == -math.inf).all()
            seen += p.view(Hkv, Hq // Hkv, -1).sum(1)
            wtol += (p * (2 * rel + 16 * U[F32])).view(Hkv, Hq // Hkv, -1).sum(1)
        if weights:
            base = torch.zeros(Hkv, total[b], dtype=torch.float64) if w_null else w_in[b, :, :total[b]].cpu().double()
            steps = (M * Hq // Hkv + 1) * U[F32]
            assert ((gw[b, :, :total[b]] - base - seen).abs() <= wtol + steps * (base + seen) + 1e-30).all(), b
            assert (gw[b, :, total[b]:] == -9).all()


def stale(pool, b, n):
    """NaN and infinities in every slot of series b's pages from slot n on."""
    page = pool.page
    for s in range(n, int((pool.table[b] >= 0).sum()) * page):
        pool.put(pool.k, b, s, math.nan if s % 2 else math.inf)
        pool.put(pool.v, b, s, math.inf if s % 2 else math.nan)


LENGTHS = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 200, 513, 3]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,Hq,Hkv,M,page,order", [
    (64, 8, 8, 1, 16, "heads"), (128, 32, 8, 1, 32, "slots"), (32, 4, 4, 1, 8, "heads"), (64, 20, 4, 9, 16, "heads"), (128, 6, 2, 5, 64, "slots"),
    (32, 12, 1, 3, 16, "slots"), (64, 3, 3, 33, 1, "heads"), (128, 7, 1, 17, 128, "heads"), (64, 16, 1, 1, 32, "slots"), (64, 34, 2, 1, 32, "slots"), (128, 3, 3, 1, 16, "heads"), (128, 2, 1, 1, 8, "slots"), (64, 2, 1, 1, 16, "heads"), (32, 4, 2, 1, 32, "heads"),
    (128, 3, 1, 1, 64, "heads"), (32, 3, 1, 2, 8, "slots"), (128, 8, 1, 1, 16, "heads")])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 20), (True, 1), (False, 70)])
def test_attention(dtype, D, Hq, Hkv, M, page, order, causal, window):
    new = [min(M, 1 + b % M) if b % 5 else M for b in range(len(LENGTHS))]
    new[4] = 0
    total = [n + (m if causal else 0) for n, m in zip(LENGTHS, new)]
    pool = Pool(len(LENGTHS), Hkv, D, page, total, dtype, order, seed=D + M)
    for b, n in enumerate(total):
        stale(pool, b, n)
    check_attention(pool, dtype, Hq, Hkv, D, LENGTHS, new, M, causal, window, weights=window != 1, qpad=8, w_null=window == 70)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,Hq,Hkv,M,lengths", [
    (128, 8, 1, 1, [40000]), (64, 4, 2, 1, [20011, 3]), (64, 10, 2, 9, [9001, 0, 130]), (128, 40, 8, 1, [1000] * 40), (32, 2, 1, 1, [5] * 700),
    (64, 2, 1, 2, list(range(300)))])
def test_attention_split_over_the_length(dtype, D, Hq, Hkv, M, lengths):
    pool = Pool(len(lengths), Hkv, D, 32, [n + M for n in lengths], dtype, seed=3)
    check_attention(pool, dtype, Hq, Hkv, D, lengths, [M] * len(lengths), M, weights=len(lengths) < 4)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,Hq,Hkv,M,page,lengths", [
    (64, 4, 2, 1, 512, [700, 3, 512, 1023]), (128, 8, 8, 2, 65536, [900]), (32, 2, 1, 1, 4, [333, 64]), (64, 1, 1, 1, 16, [b % 7 for b in range(3000)]),
    (128, 96, 2, 1, 32, [500, 64]), (64, 8, 1, 5, 2, [130, 0, 64])])
def test_attention_over_pages_of_any_size_and_many_series(dtype, D, Hq, Hkv, M, page, lengths):
    """Pages longer than a tile, of less than a copied box, one that holds everything; thousands of series; more rows than a CTA takes at once."""
    pool = Pool(len(lengths), Hkv, D, page, [n + M for n in lengths], dtype, seed=6)
    for b in (0, len(lengths) - 1):
        stale(pool, b, min(lengths[b] + M, int((pool.table[b] >= 0).sum()) * page - 200) if page > 1000 else lengths[b] + M)
    check_attention(pool, dtype, Hq, Hkv, D, lengths, [M] * len(lengths), M, weights=len(lengths) < 10)


def test_two_streams_with_workspaces_of_their_own():
    """Calls that overlap on the GPU: each gives what it gives alone."""
    tsfm = lib()
    B, Hq, Hkv, D, n = 8, 16, 4, 64, 6000
    pool = Pool(B, Hkv, D, 32, [n] * B, BF16, seed=12)
    pages = pool.describe(tsfm)
    size = tsfm.tsfm_paged_attention_workspace(pages, B, 1, Hq, n)
    q = [wide((B, 1), Hq * D, BF16, 0, 20 + i) for i in range(2)]
    length = [ints([n - 500 * b * i for b in range(B)]) for i in (1, 0)]
    work = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def attend(i, out):
        tsfm.tsfm_paged_attention(stream(), pages, q[i], Hq * D, out, Hq * D, length[i], None, B, 1, Hq, 0.125, False, 0, n, None, None, None, 0, work[i], size)
    alone = [torch.empty_like(q[0]) for _ in range(2)]
    for i in range(2):
        attend(i, alone[i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        outs = [torch.zeros_like(q[0]) for _ in range(2)]
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                attend(i, outs[i])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], alone[0]) and torch.equal(outs[1], alone[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_with_peaked_and_shifted_scores(dtype):
    """Scores around +-1000 with one slot far above the rest: the running maximum, not the scores' size, sets the range."""
    B, Hkv, D = 3, 2, 64
    pool = Pool(B, Hkv, D, 16, [300, 77, 150], dtype, seed=5)
    for b, n in enumerate([299, 0, 100]):
        pool.put(pool.k, b, n, 6.0)
    check_attention(pool, dtype, 4, Hkv, D, [299, 76, 149], [1, 1, 1], 1, scale=4.0, weights=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,Hq", [(9, 4), (3, 2), (5, 16)])
def test_a_later_token_that_is_not_finite_stays_unseen(dtype, M, Hq):
    """Each new token's key and value are NaN or infinite: the tokens before it are as if it did not exist, those from it on are not
    finite.  The same for old slots that a window leaves out for some of the tokens only."""
    tsfm = lib()
    B, Hkv, D, n = 2, 2, 64, 70
    for window in (0, 40):
        for bad, slot in ((1, n + 1), (2, n + M - 1), (1, n - 39)):
            pool = Pool(B, Hkv, D, 16, [n + M] * B, dtype, seed=bad)
            clean_v, clean_k = pool.v.clone(), pool.k.clone()
            pool.put(pool.v, 0, slot, math.nan if bad == 1 else math.inf)
            q = wide((B, M), Hq * D, dtype, 0, 4)
            got = []
            for k, v in ((clean_k, clean_v), (pool.k, pool.v)):
                pages = tsfm.kv_pages(k, v, pool.table)
                out = torch.zeros(B, M, Hq * D, dtype=dtype, device="cuda")
                work = torch.empty(tsfm.tsfm_paged_attention_workspace(pages, B, M, Hq, n + M), dtype=torch.uint8, device="cuda")
                tsfm.tsfm_paged_attention(stream(), pages, q, q.stride(1), out, out.stride(1), ints([n] * B), None, B, M, Hq, 0.1, True, window, n + M,
                                          None, None, None, 0, work, work.numel())
                got.append(out.cpu())
            for m in range(M):
                sees = slot <= n + m and (not window or slot > n + m - window)
                if sees:
                    assert not torch.isfinite(got[1][0, m]).any(), (window, bad, slot, m)
                else:
                    assert torch.equal(got[0][0, m], got[1][0, m]), (window, bad, slot, m)
            assert torch.equal(got[0][1], got[1][1])


def test_attention_hides_pages_outside_the_pool_and_reports_them():
    tsfm = lib()
    for dtype in (F32, BF16):
        pool = Pool(2, 2, 64, 16, [64, 64], dtype, seed=9)
        whole = pool.table.clone()
        pool.table[1, 1:] = pool.k.shape[0] + 5                # series 1: only its first 16 slots
        args = dict(lse=torch.zeros(2, 1, 4, device="cuda"), out=torch.zeros(2, 1, 256, dtype=dtype, device="cuda"))
        q = wide((2, 1), 256, dtype, 0, 2)
        got = []
        for table, length in ((pool.table, [64, 64]), (whole, [64, 16])):
            pages = pool.describe(tsfm, table)
            work = torch.empty(tsfm.tsfm_paged_attention_workspace(pages, 2, 1, 4, 64), dtype=torch.uint8, device="cuda")
            tsfm.tsfm_paged_attention(stream(), pages, q, 256, args["out"], 256, ints(length), None, 2, 1, 4, 0.125, False, 0, 64, args["lse"], None, None, 0,
                                      work, work.numel())
            got.append((args["out"].cpu().double(), args["lse"].cpu().double(), int(pool.status)))
            pool.status.zero_()
        assert got[0][2] == tsfm.TSFM_PAGES_BAD_ID and got[1][2] == 0
        assert (got[0][0] - got[1][0]).abs().max() <= 4 * U[dtype] * got[1][0].abs().max() and (got[0][1] - got[1][1]).abs().max() < 1e-5
        # lengths beyond the capacity or below 0 are cut
        check_attention(Pool(1, 2, 64, 16, [64], dtype, seed=1), dtype, 4, 2, 64, [64], [1], 1, causal=False, max_len=64)
        pool = Pool(3, 2, 64, 16, [64, 64, 64], dtype, seed=2)
        pages = pool.describe(tsfm)
        work = torch.empty(tsfm.tsfm_paged_attention_workspace(pages, 3, 1, 4, 50), dtype=torch.uint8, device="cuda")
        out = [torch.zeros(3, 1, 256, dtype=dtype, device="cuda") for _ in range(2)]
        q = wide((3, 1), 256, dtype, 0, 2)
        for o, length in zip(out, ([1 << 30, -5, 50], [50, 0, 50])):
            tsfm.tsfm_paged_attention(stream(), pages, q, 256, o, 256, ints(length), None, 3, 1, 4, 0.125, False, 0, 50, None, None, None, 0, work, work.numel())
        assert torch.equal(out[0], out[1]) and (out[0][1] == 0).all() and int(pool.status) == tsfm.TSFM_PAGES_BAD_LEN


def test_attention_is_the_same_each_time_and_lets_its_weights_accumulate_in_place():
    tsfm = lib()
    B, M, Hq, Hkv, D, n = 7, 3, 8, 2, 64, 1500
    pool = Pool(B, Hkv, D, 32, [n] * B, BF16, seed=4)
    length = ints([n - M - 100 * b for b in range(B)])
    pages = pool.describe(tsfm)
    work = torch.empty(tsfm.tsfm_paged_attention_workspace(pages, B, M, Hq, n, True), dtype=torch.uint8, device="cuda")
    q = wide((B, M), Hq * D, BF16, 0, 7)
    first = None
    for i in range(6):
        out, w = torch.zeros(B, M, Hq * D, dtype=BF16, device="cuda"), torch.ones(B, Hkv, n, device="cuda")
        work.random_(0, 256)
        w_in = w if i % 2 else torch.ones_like(w)
        tsfm.tsfm_paged_attention(stream(), pages, q, q.stride(1), out, out.stride(1), length, None, B, M, Hq, 0.125, True, 0, n, None, w_in, w, n, work, work.numel())
        if first is None:
            first = (out, w)
        assert torch.equal(out, first[0]) and torch.equal(w, first[1])
    total = (length[:, None] + M).expand(B, Hkv)
    got = (first[1] - 1).double().cpu().sum(2)                 # every row's probabilities add up to 1
    assert (got - M * Hq / Hkv).abs().max() < 1e-3 and int(total.min()) > 0


# ------------------------------------------------------------------------------------------ eviction
def check_evict(B, Hkv, D, page, lengths, budget, sinks, recent, dtype, w, order="heads", max_len=None):
    tsfm = lib()
    max_len = max_len or max(1, max(lengths))
    kept_n = [min(n, budget) for n in lengths]
    need = sum(-(-n // page) for n in kept_n)
    pool = Pool(B, Hkv, D, page, lengths, dtype, order, seed=budget, spare=need + 1)
    dst = torch.full((B, max(1, -(-min(budget, max_len) // page))), -1, dtype=torch.int32)
    ids = list(pool.spare_ids)
    for b, n in enumerate(kept_n):
        for i in range(-(-n // page)):
            dst[b, i] = ids.pop()
    dst = dst.cuda()
    k0, v0 = pool.k.clone(), pool.v.clone()
    kept = torch.full((B, Hkv, budget), -5, dtype=torch.int32, device="cuda")
    w_out = torch.full((B, Hkv, budget + 2), -5.0, device="cuda")
    len_out = torch.full((B,), -5, dtype=torch.int32, device="cuda")
    wd = w.cuda()
    tsfm.tsfm_cache_evict(stream(), pool.describe(tsfm), dst, dst.shape[1], ints(lengths), wd, wd.shape[2], B, budget, sinks, recent, max_len, kept, w_out,
                          budget + 2, len_out)
    torch.cuda.synchronize()
    assert int(pool.status) == 0 and len_out.tolist() == kept_n
    want_k, want_v = k0.clone(), v0.clone()
    for b, n in enumerate(lengths):
        for h in range(Hkv):
            slots = ref.evict(w[b, h].tolist(), n, budget, sinks, recent)
            assert kept[b, h].tolist() == slots + [-1] * (budget - len(slots)), (b, h)
            idx = torch.tensor(slots, dtype=torch.long)
            assert torch.equal(w_out[b, h, :len(slots)].cpu().view(torch.int32), w[b, h, idx].view(torch.int32))
            assert (w_out[b, h, len(slots):] == -5).all()
            if slots:
                j = torch.arange(len(slots))
                src, to = pool.table[b].cpu()[idx // page].long().cuda(), dst[b].cpu()[j // page].long().cuda()
                for want, old in ((want_k, k0), (want_v, v0)):
                    want[to, h, (j % page).cuda()] = old[src, h, (idx % page).cuda()]
    assert torch.equal(pool.k, want_k) and torch.equal(pool.v, want_v)


@pytest.mark.parametrize("dtype,D,page,order", [(BF16, 128, 16, "heads"), (F32, 64, 32, "slots"), (BF16, 32, 8, "heads"), (F32, 128, 1, "heads")])
@pytest.mark.parametrize("lengths,budget,sinks,recent", [
    ([100, 64, 65, 0, 1, 63], 64, 4, 16), ([500, 33], 40, 0, 0), ([300], 299, 10, 20), ([77, 80], 50, 20, 30), ([2049, 4100], 1000, 4, 0), ([9], 1, 0, 0),
    ([9], 1, 1, 0), ([9], 1, 0, 1), ([30, 2], 4096, 4, 8)])
def test_evict(dtype, D, page, order, lengths, budget, sinks, recent):
    B, Hkv = len(lengths), 3
    g = torch.Generator().manual_seed(budget)
    w = torch.rand(B, Hkv, max(lengths) + 5, generator=g)
    w[:, 1] = (w[:, 1] * 4).floor()                            # many ties
    w[:, 2, ::3] = -w[:, 2, ::3]
    check_evict(B, Hkv, D, page, lengths, budget, sinks, recent, dtype, w, order)


def test_evict_orders_all_floats():
    """Ties, signed zeros, infinities, NaN, subnormals, values that differ in their last bit."""
    n, specials = 1200, [0.0, -0.0, math.inf, -math.inf, math.nan, 1e-45, -1e-45, 1.0, 1.0 + 2.0 ** -23, 3.4e38, -3.4e38]
    g = torch.Generator().manual_seed(0)
    w = torch.tensor(specials)[torch.randint(len(specials), (1, 4, n), generator=g)]
    w[0, 3] = torch.randint(-2 ** 31, 2 ** 31 - 1, (n,), generator=g, dtype=torch.int64).int().view(F32)
    for budget in (1, 50, 300, 600, 1000, 1199):
        check_evict(1, 4, 32, 16, [n], budget, 0, 0, F32, w)


def test_evict_long_and_wrong_pages():
    tsfm = lib()
    g = torch.Generator().manual_seed(1)
    check_evict(1, 2, 64, 64, [70001], 30011, 4, 500, BF16, torch.rand(1, 2, 70001, generator=g))
    check_evict(2, 1, 32, 64, [140001, 5], 1000, 4, 500, BF16, torch.rand(2, 1, 140001, generator=g))         # beyond a cluster's shared memory
    check_evict(3, 2, 32, 16, [16385, 5000, 8193], 4095, 0, 1, F32, (torch.rand(3, 2, 16385, generator=g) * 50).floor())
    # a wrong page id: what lies there is not moved, the rest is
    pool = Pool(1, 1, 32, 8, [32], F32, seed=2, spare=2)
    table, dst = pool.table.clone(), ints([[pool.spare_ids[0], 99]])
    table[0, 1] = 1 << 20
    w = torch.arange(32, 0, -1).float().view(1, 1, 32).cuda()  # keeps slots 0..15
    kept, len_out = ints([[[0] * 16]]), ints([0])
    before = pool.k.clone()
    tsfm.tsfm_cache_evict(stream(), pool.describe(tsfm, table), dst, 2, ints([40]), w, 32, 1, 16, 0, 0, 32, kept, None, 0, len_out)
    assert int(pool.status) == tsfm.TSFM_PAGES_BAD_ID | tsfm.TSFM_PAGES_BAD_LEN and len_out.tolist() == [16] and kept[0, 0].tolist() == list(range(16))
    before[pool.spare_ids[0]] = before[table[0, 0].long()]
    assert torch.equal(pool.k, before)


# ------------------------------------------------------------------------------------------ verification
def check_verify(tokens, p, q, u, nd=None, lens=None, ppad=0, qpad=0, seed=0, rnd=0, s0=0, alias=False):
    tsfm = lib()
    B, K1, V = p.shape
    K = K1 - 1

    def padded(x, pad):
        if x is None:
            return None
        y = torch.full((*x.shape[:-1], V + pad), math.nan)
        y[..., :V] = x
        return y.cuda()
    pd, qd = padded(p, ppad), padded(q, qpad)
    out = torch.full((B, K + 1), -7, dtype=torch.int32, device="cuda")
    n_acc = ints([-7] * B)
    len_in = ints(lens) if lens is not None else None
    len_out = None if lens is None else len_in if alias else torch.zeros_like(len_in)
    tsfm.tsfm_verify_tokens(stream(), None if K == 0 else tokens.int().cuda(), pd, V + ppad, qd, V + qpad, B, K, V, None if u is None else u.cuda(), seed, rnd, s0,
                            None if nd is None else ints(nd), len_in, out, n_acc, len_out)
    torch.cuda.synchronize()
    for b in range(B):
        ub = u[b].numpy() if u is not None else np.array([orc.acceptance_uniform(seed, s0 + b, rnd, i) for i in range(K + 1)], np.float32)
        n_d = K if nd is None else min(max(nd[b], 0), K)
        want, n = ref.verify(tokens[b].numpy() if K else [], p[b].numpy(), None if q is None else q[b].numpy(), ub, n_d)
        assert n_acc[b].item() == n, b
        assert out[b].tolist() == want + [-1] * (K + 1 - len(want)), (b, n)
        if lens is not None:
            assert len_out[b].item() == lens[b] + n + 1


def distributions(B, K, V, seed, sharp=2.0, apart=0.5, cut=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, K + 1, V, generator=g) * sharp
    soft = lambda x: torch.where((p := torch.softmax(x, -1)) < cut / V, torch.zeros_like(p), p)
    q, p = soft(x[:, :K]), soft(x + apart * torch.randn(x.shape, generator=g))
    tokens = torch.multinomial(q.reshape(-1, V), 1, generator=g).view(B, K) if K else torch.zeros(B, 0)
    return tokens, p, q, torch.rand(B, K + 1, generator=g)


@pytest.mark.parametrize("B,K,V,cut", [(1, 4, 32003, 0.0), (64, 8, 1000, 0.1), (300, 3, 513, 0.0), (7, 32, 100, 0.1), (3, 5, 100003, 0.0), (40, 2, 16385, 0.2),
                                       (1, 1, 131072, 0.0), (300, 1, 100003, 0.3), (20, 4, 1, 0.0), (50, 4, 2, 0.0), (9, 4, 31, 0.0), (2, 0, 5000, 0.0), (148, 1, 4097, 0.0)])
@pytest.mark.parametrize("sampled", [True, False])
def test_verify_tokens(B, K, V, cut, sampled):
    tokens, p, q, u = distributions(B, K, V, B + V, cut=cut)
    if not sampled:
        tokens = q.argmax(-1) if K else tokens
    nd = None if B % 2 else [(b * 3) % (K + 2) - 1 + (b % 5 == 0) * K for b in range(B)]
    check_verify(tokens, p, q if sampled and K else None, u, nd, lens=list(range(B)), ppad=B % 4, qpad=B % 3, alias=bool(B % 2))


def test_verify_uniforms_at_their_ends_and_wrong_values():
    """u 0, just below 1, 1, above, negative, NaN; tokens outside the vocabulary; p equal to q; probabilities that are 0, negative, NaN or infinite."""
    V, K = 700, 3
    ends = [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, math.nan, 2.0 ** -149]
    B = len(ends) * 6
    tokens, p, q, u = distributions(B, K, V, 5)
    u = torch.tensor(ends).repeat_interleave(6)[:, None].expand(B, K + 1).contiguous()
    for b in range(B):
        if b % 6 == 0:
            p[b, :K] = q[b]                                    # always accepted
        if b % 6 == 1:
            tokens[b, 1] = (-1, V, 2 ** 31 - 1, -2 ** 31)[b // 6 % 4]
        if b % 6 == 2:
            p[b, 0, tokens[b, 0]] = 0.0                        # never accepted, not even with u = 0
        if b % 6 == 3:
            p[b, 0] = torch.minimum(p[b, 0], q[b, 0]) * 0.5    # p nowhere above q: the draw is from p
        if b % 6 == 4:
            p[b, :, ::7], p[b, :, 1::7], p[b, :, 2::7] = math.nan, math.inf, -1.0
            q[b, :, ::5] = math.nan
        if b % 6 == 5:
            p[b, 1] = 0.0                                      # nothing to draw from
    check_verify(tokens, p, q, u)
    check_verify(q.nan_to_num(0).argmax(-1), p, None, u)


@pytest.mark.parametrize("V", [3, 1000, 20000, 90001])
def test_verify_draws_at_the_borders_of_the_distribution(V):
    """Uniforms at and next to k / 8 of distributions of eight equal entries, in runs of zeros anywhere: borders are exact in fp64."""
    g = torch.Generator().manual_seed(V)
    n = min(8, V) if V < 8 else 8
    n = 2 if V == 3 else n
    B = 3 * n
    p, u = torch.zeros(B, 1, V), torch.zeros(B, 1)
    for b in range(B):
        at = torch.randperm(V, generator=g)[:n]
        p[b, 0, at] = 0.125
        border = (b // 3) / n
        u[b, 0] = [border, max(0.0, border - 2.0 ** -24), border + 2.0 ** -24][b % 3]
    check_verify(torch.zeros(B, 0), p, None, u)


@pytest.mark.parametrize("B,K,V", [(6, 4, 300), (200, 2, 40), (1, 3, 50000)])
def test_verify_draws_its_own_uniforms_as_the_accept_step_does(B, K, V):
    tokens, p, q, _ = distributions(B, K, V, 11)
    check_verify(tokens, p, q, None, seed=2021 + (9 << 32), rnd=4, s0=17)


# ------------------------------------------------------------------------------------------ together
def test_offsets_beyond_32_bits():
    """Pages whose bytes and whose elements lie behind 2^32: append, attention and eviction over them."""
    tsfm = lib()
    Hkv, page, D, n_pages = 8, 64, 128, 66000                  # 64 Ki elements a page: 4.3e9 of them, 8.7 GB a pool
    k = torch.zeros(n_pages, Hkv, page, D, dtype=BF16, device="cuda")
    v = torch.zeros(n_pages, Hkv, page, D, dtype=BF16, device="cuda")
    n, M, Hq = 150, 2, 8
    table, dst = ints([[n_pages - 1, 3, n_pages - 2]]), ints([[n_pages - 3, n_pages - 4]])
    pages = tsfm.kv_pages(k, v, table)
    qkv = wide((1, n), (Hq + 2 * Hkv) * D, BF16, 0, 8)
    rope, f = make_rope("half", D, "plain")
    q = torch.zeros(1, n, Hq * D, dtype=BF16, device="cuda")
    tsfm.tsfm_rope_append(stream(), rope, pages, qkv, qkv.stride(1), q, q.stride(1), None, ints([0]), None, 1, n, Hq)
    slots = torch.arange(n)
    at = table[0].cpu()[slots // page].long().cuda()
    kk, vv = k[at, :, (slots % page).cuda()].cpu().double(), v[at, :, (slots % page).cuda()].cpu().double()
    assert torch.equal(vv, qkv[0].cpu().double().view(n, -1, D)[:, Hq + Hkv:])
    for s in (0, 64, 149):
        want = ref.turn(qkv[0, s].cpu().double().view(-1, D)[Hq:Hq + Hkv], float(s), f, "half")
        assert (kk[s] - want).abs().max() <= (U[BF16] + 2.0 ** -20) * want.abs().max()
    out, lse = torch.zeros(1, M, Hq * D, dtype=BF16, device="cuda"), torch.zeros(1, M, Hq, device="cuda")
    w = torch.zeros(1, Hkv, n, device="cuda")
    work = torch.empty(tsfm.tsfm_paged_attention_workspace(pages, 1, M, Hq, n, True), dtype=torch.uint8, device="cuda")
    tail = q[:, n - M:]
    tsfm.tsfm_paged_attention(stream(), pages, tail, tail.stride(1), out, out.stride(1), ints([n - M]), None, 1, M, Hq, D ** -0.5, True, 0, n, lse, None, w, n, work, work.numel())
    for m in range(M):
        o, z, _, absv, peak = ref.attention(tail[0, m].cpu().double().view(Hq, D), kk, vv, D ** -0.5, 0, n - M + m + 1)
        rel = ref.attention_tolerance(BF16, D, n, peak)[:, None]
        assert ((out[0, m].cpu().double().view(Hq, D) - o).abs() <= U[BF16] * o.abs() + rel * absv).all()
    kept, len_out = torch.zeros(1, Hkv, 100, dtype=torch.int32, device="cuda"), ints([0])
    tsfm.tsfm_cache_evict(stream(), pages, dst, 2, ints([n]), w, n, 1, 100, 4, 20, n, kept, None, 0, len_out)
    for h in range(Hkv):
        slots = ref.evict(w[0, h].tolist(), n, 100, 4, 20)
        assert kept[0, h].tolist() == slots
        j = torch.arange(100)
        to = dst[0].cpu()[j // page].long().cuda()
        assert torch.equal(k[to, h, (j % page).cuda()].cpu().double(), kk[slots, h]) and torch.equal(v[to, h, (j % page).cuda()].cpu().double(), vv[slots, h])


class Loop:
    """A served model of one attention layer over quantised values: fixed random maps around the calls under test, fp32."""

    def __init__(self, B, K, V, Hq, Hkv, D, page, slots, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.K, self.V, self.Hq, self.Hkv, self.D, self.page, self.slots = B, K, V, Hq, Hkv, D, page, slots
        self.emb = (torch.randn(V, (Hq + 2 * Hkv) * D, generator=g) * 0.7).cuda()
        self.head = (torch.randn(Hq * D, V, generator=g) * 0.25).cuda()
        self.pool = Pool(B, Hkv, D, page, [slots] * B, F32, seed=seed, fill=0.0, spare=B * -(-slots // page))
        self.other = ints([self.pool.spare_ids[b::B] for b in range(B)])
        self.rope, self.f = make_rope("half", D, "plain")
        self.len = ints([0] * B)
        self.pos = ints([0] * B)
        self.w = torch.zeros(B, Hkv, slots, device="cuda")
        self.tokens = torch.zeros(B, K + 1, dtype=torch.int32, device="cuda")
        self.draft = torch.zeros(B, K, dtype=torch.int32, device="cuda")
        self.u = torch.zeros(B, K + 1, device="cuda")
        self.q_out = torch.zeros(B, K + 1, Hq * D, device="cuda")
        self.att = torch.zeros(B, K + 1, Hq * D, device="cuda")
        self.lse = torch.zeros(B, K + 1, Hq, device="cuda")
        self.out = torch.zeros(B, K + 1, dtype=torch.int32, device="cuda")
        self.n_acc = ints([0] * B)
        self.p = torch.zeros(B, K + 1, V, device="cuda")
        tsfm = lib()
        self.pages = self.pool.describe(tsfm)
        self.work = torch.empty(tsfm.tsfm_paged_attention_workspace(self.pages, B, K + 1, Hq, slots, True), dtype=torch.uint8, device="cuda")

    def round(self):
        """The pending token and K drafted ones in self.tokens: append, attend, verify; lengths move on."""
        tsfm, B, M = lib(), self.B, self.K + 1
        qkv = self.emb[self.tokens.long()]
        tsfm.tsfm_rope_append(stream(), self.rope, self.pages, qkv, qkv.stride(1), self.q_out, self.q_out.stride(1), self.pos, self.len, None, B, M, self.Hq)
        tsfm.tsfm_paged_attention(stream(), self.pages, self.q_out, self.q_out.stride(1), self.att, self.att.stride(1), self.len, None, B, M, self.Hq,
                                  self.D ** -0.5, True, 0, self.slots, self.lse, self.w, self.w, self.slots, self.work, self.work.numel())
        torch.softmax(self.att @ self.head, -1, out=self.p)
        self.draft.copy_(self.tokens[:, 1:])
        tsfm.tsfm_verify_tokens(stream(), self.draft, self.p, self.V, None, 0, B, self.K, self.V, self.u, 0, 0, 0, None, self.len, self.out, self.n_acc, self.len)
        self.pos += self.n_acc + 1


def test_rounds_of_a_served_model_with_rollback_and_eviction():
    """Append, attend, verify and roll back, evict, go on: every round against a recomputation in 64 bits from the committed tokens and the
    slots that were kept."""
    tsfm = lib()
    B, K, V, Hq, Hkv, D, page, slots, budget = 3, 3, 60, 4, 2, 32, 8, 64, 24
    L = Loop(B, K, V, Hq, Hkv, D, page, slots)
    g = torch.Generator().manual_seed(3)
    pending = [1, 2, 3]
    cache = [[[] for _ in range(Hkv)] for _ in range(B)]       # what each head holds: (token, position)
    position = [0] * B
    acc = [[{} for _ in range(Hkv)] for _ in range(B)]         # accumulated weight and its tolerance by position
    emb = L.emb.cpu().double().view(V, Hq + 2 * Hkv, D)
    accepted = 0
    for r in range(14):
        draft = torch.randint(0, V, (B, K), generator=g)
        if r:                                                  # drafts that pass now and then: the target's own favourites
            draft[:, 0] = L.p[torch.arange(B), L.n_acc.long()].argmax(-1).cpu()
        L.tokens.copy_(torch.cat([torch.tensor(pending)[:, None], draft], 1).int())
        L.u.copy_(torch.rand(B, K + 1, generator=g) * torch.tensor([0.05] * K + [1.0]))
        L.round()
        torch.cuda.synchronize()
        p, att = L.p.cpu(), L.att.cpu().double()
        for b in range(B):
            toks = [pending[b]] + draft[b].tolist()
            for h in range(Hkv):
                hold = cache[b][h] + [(t, position[b] + i) for i, t in enumerate(toks)]
                k = torch.stack([ref.turn(emb[t, Hq + h:Hq + h + 1], float(x), L.f, "half")[0] for t, x in hold])[:, None]
                v = torch.stack([emb[t, Hq + Hkv + h] for t, _ in hold])[:, None]
                for m, t in enumerate(toks):
                    qs = ref.turn(emb[t, h * 2:h * 2 + 2], float(position[b] + m), L.f, "half")
                    end = len(cache[b][h]) + m + 1
                    o, _, pr, absv, peak = ref.attention(qs, k, v, D ** -0.5, 0, end)
                    # the cached keys and the queries are rounded to 32 bits, as their angles are: 2^-20 of a score's terms
                    rel = (ref.attention_tolerance(F32, D, end, peak) + 2.0 ** -19 * peak)[:, None]
                    assert ((att[b, m].view(Hq, D)[2 * h:2 * h + 2] - o).abs() <= rel * absv + 4 * U[F32] * o.abs()).all(), (r, b, h, m)
                    for (_, x), wt, off in zip(hold[:end], pr.sum(0).tolist(), (pr * (2 * rel + 16 * U[F32])).sum(0).tolist()):
                        w0, t0 = acc[b][h].get(x, (0.0, 0.0))
                        acc[b][h][x] = (w0 + wt, t0 + off)
            want, n = ref.verify(draft[b].numpy(), p[b].numpy(), None, L.u[b].cpu().numpy(), K)
            assert L.out[b, :n + 1].tolist() == want and int(L.n_acc[b]) == n
            accepted += n
            for h in range(Hkv):
                cache[b][h] += [(t, position[b] + i) for i, t in enumerate(toks[:n + 1])]
                for i in range(n + 1, K + 1):                  # weight that rejected tokens got is not theirs to keep
                    acc[b][h].pop(position[b] + i, None)
            position[b] += n + 1
            pending[b] = want[-1]
        # slots behind the committed length start from 0 again
        behind = torch.arange(slots, device="cuda") >= L.len[:, None, None]
        L.w.masked_fill_(behind, 0.0)
        assert L.len.tolist() == [len(cache[b][0]) for b in range(B)] and L.pos.tolist() == position
        if r % 5 == 4:
            table, k_len = L.pool.table, L.len.clone()
            kept, w_new = torch.zeros(B, Hkv, budget, dtype=torch.int32, device="cuda"), torch.zeros_like(L.w)
            w_host = L.w.cpu()
            len_out = torch.zeros_like(L.len)
            tsfm.tsfm_cache_evict(stream(), L.pages, L.other, L.other.shape[1], L.len, L.w, slots, B, budget, 2, 6, slots, kept, w_new, slots, len_out)
            torch.cuda.synchronize()
            for b in range(B):
                for h in range(Hkv):
                    n = int(k_len[b])
                    for s, (_, x) in enumerate(cache[b][h]):
                        want, off = acc[b][h][x]           # (a sum of up to 14 rounds of 8 probabilities)
                        assert abs(float(w_host[b, h, s]) - want) <= off + 14 * 9 * U[F32] * want
                    slots_kept = ref.evict(w_host[b, h].tolist(), n, budget, 2, 6)
                    assert kept[b, h, :len(slots_kept)].tolist() == slots_kept
                    cache[b][h] = [cache[b][h][s] for s in slots_kept]
            L.len.copy_(len_out)
            L.w.copy_(w_new)
            L.pool.table, L.other = L.other, table
            L.pages = L.pool.describe(tsfm)
    assert accepted > 5 and int(L.pool.status) == 0 and max(position) > budget


def test_rounds_captured_in_a_graph_repeat_the_eager_ones():
    """One captured round, replayed with new tokens and uniforms, on another stream than the eager one."""
    results = []
    for graph in (False, True):
        L = Loop(5, 4, 200, 8, 2, 64, 16, 128, seed=1)
        g = torch.Generator().manual_seed(8)
        captured, side = None, torch.cuda.Stream()
        seen = []
        for r in range(8):
            L.tokens.copy_(torch.randint(0, 200, (5, 5), generator=g).int())
            L.u.copy_(torch.rand(5, 5, generator=g) * torch.tensor([0.02] * 4 + [1.0]))
            torch.cuda.synchronize()
            if not graph:
                L.round()
            else:
                if captured is None:
                    with torch.cuda.stream(side):                # a first pass for the products' own set-up, then from the start again
                        state = [t.clone() for t in (L.len, L.pos, L.w)]
                        L.round()
                        for t, s in zip((L.len, L.pos, L.w), state):
                            t.copy_(s)
                    torch.cuda.synchronize()
                    captured = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(captured, stream=side):
                        L.round()
                captured.replay()
            torch.cuda.synchronize()
            seen.append([t.clone() for t in (L.att, L.out, L.n_acc, L.len, L.w)])
        results.append(seen)
        del captured
    for a, b in zip(*results):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
