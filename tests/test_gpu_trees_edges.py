"""Attention of trees and windows, log probabilities: batches, masks, values and scales that the ordinary cases (tests/test_gpu_trees.py) leave out."""
import math

import numpy as np
import pytest
import torch

from tests import serving_ref as ref
from tests import trees_ref as tr
from tests.serving_ref import U, Pool
from tests.test_gpu_serving import ints, lib, stale, stream, wide
from tests.test_gpu_trees import BF16, F32, check, check_logprobs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,M,Hq", [(64, 70, 32), (128, 61, 32), (64, 150, 16)])
def test_long_units_beside_short_ones(D, M, Hq):
    """Units of more than 128 live rows and of fewer, in turn, long ones behind short ones and the other way round, many for each CTA: those of its warps
    that have no rows in a unit come back in the next.  The same answer each time."""
    B, Hkv = 20, 8
    lengths = [(37, 700, 64, 390, 1)[b % 5] for b in range(B)]
    new = [(M, 3, M - 1, 2 * 128 * Hkv // Hq // 3, M, 0)[b % 6] for b in range(B)]
    pool = Pool(B, Hkv, D, 16, [n + m for n, m in zip(lengths, new)], BF16, seed=1)
    for b in range(B):
        stale(pool, b, lengths[b] + new[b])
    trees = [tr.tree("random", M, b) for b in range(B)]
    for window, sinks in ((0, 0), (50, 3)):
        a = check(pool, BF16, Hq, Hkv, D, lengths, new, M, trees, window=window, sinks=sinks, seed=2)
        again = check(pool, BF16, Hq, Hkv, D, lengths, new, M, trees, window=window, sinks=sinks, seed=2, runs=10)
        assert all(torch.equal(x, y) for x, y in zip(a, again))


@pytest.mark.parametrize("D,Hq,M", [(64, 8, 40), (128, 8, 20), (64, 16, 70)])
@pytest.mark.parametrize("miss_from", [0, 1])
def test_a_wait_that_runs_out_in_a_short_run(D, Hq, M, miss_from):
    """Runs of one or two tiles: the warp that fetches has asked for all of them and meets no wait that runs out, the others do.  The call ends, says so, and
    the next one is whole."""
    tsfm = lib()
    lengths = [3, 100, 128, 60]
    pool = Pool(4, 2, D, 16, [n + M for n in lengths], BF16, seed=3)
    q = wide((4, M), Hq * D, BF16, 0, 1)
    pages = pool.describe(tsfm)
    mask, depth = tr.ancestors(tr.tree("random", M, 1))
    mask, depth = tr.words(mask).cuda(), ints(depth)
    size = tsfm.tsfm_tree_attention_workspace(pages, 4, M, Hq, 128 + M)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def run():
        out = torch.zeros_like(q)
        tsfm.tsfm_tree_attention(stream(), pages, q, q.stride(1), out, out.stride(1), ints(lengths), None, mask, depth, True, 4, M, Hq, 0.125, 0, 0, 128 + M, None, ws,
                                 size)
        torch.cuda.synchronize()
        return out

    good = run()
    try:
        tsfm.tsfm_debug_tile_wait(2000, miss_from)
        bad = run()
    finally:
        tsfm.tsfm_debug_tile_wait()
    # (series 0 has one tile: nothing is missed in it from a second one on, unless its CTA has another unit's before)
    assert miss_from or (int(pool.status) == tsfm.TSFM_PAGES_TIMEOUT and torch.isnan(bad.float()).all())
    assert torch.isnan(bad.float()).any() == (int(pool.status) != 0)
    pool.status.zero_()
    assert torch.equal(run(), good) and int(pool.status) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,M,Hq", [(64, 9, 2), (32, 30, 4), (64, 26, 4), (128, 20, 8), (64, 80, 8), (128, 150, 4)])
def test_values_that_are_not_finite_spoil_their_columns_alone(dtype, D, M, Hq):
    """Some elements of some values are not finite, in tiles that every token sees whole and in others: log-sums and all other columns are those of a cache with 0
    there; tokens that see the element get no number in its column, others no trace of it."""
    tsfm = lib()
    Hkv, lengths = 2, [300, 150, 20]
    parent = [tr.tree("random", M, 5), tr.tree("star", M, 0), tr.tree("chain", M, 0)]
    pool = Pool(3, Hkv, D, 16, [n + M for n in lengths], dtype, seed=3)
    for b, n in enumerate(lengths):
        stale(pool, b, n + M)
    # slots: among the sinks; of windows; the last before the new tokens; some of these
    bad = {(0, 3, 1): {0: math.nan, D - 1: math.inf}, (0, 68, 0): {5: -math.inf}, (0, 215, 1): {D // 2: math.inf}, (0, 299, 0): {D // 2 - 1: math.nan},
           (0, 300, 1): {7: math.nan}, (0, 300 + M - 2, 0): {9: math.nan, 10: math.nan}, (1, 149, 1): {1: math.nan}, (1, 150 + M // 2, 1): {1: math.inf, 31: math.nan},
           (2, 20, 0): {c: math.nan for c in range(D)}, (2, 25, 1): {0: -math.inf}}
    clean = pool.v.clone()
    for (b, s, h), columns in bad.items():
        at = pool.table[b, s // 16].long(), h, s % 16
        for c, x in columns.items():
            pool.v[at][c], clean[at][c] = x, 0.0
    q = wide((3, M), Hq * D, dtype, 0, 1, 2.0)
    out, lse = torch.zeros_like(q), torch.zeros(3, M, Hq, device="cuda")
    pages = pool.describe(tsfm)
    work = torch.empty(tsfm.tsfm_tree_attention_workspace(pages, 3, M, Hq, 300 + M), dtype=torch.uint8, device="cuda")
    for masks, window, sinks in ((None, 100, 70), ([tr.ancestors(p) for p in parent], 0, 0), ([tr.ancestors(p) for p in parent], 100, 4), (None, 0, 0)):
        args = (stream(), pages, q, q.stride(1), out, out.stride(1), ints(lengths), None)
        rest = (3, M, Hq, 0.125, window, sinks, 300 + M, lse, work, work.numel())
        if masks:
            bits, depth = torch.stack([tr.words(s) for s, _ in masks]).cuda(), ints(np.stack([d for _, d in masks]))
            tsfm.tsfm_tree_attention(*args, bits, depth, False, *rest)
        else:
            tsfm.tsfm_window_attention(*args, *rest)
        spoiled_rows = 0
        for b, n in enumerate(lengths):
            k, v = pool.rows(pool.k, b, n + M), pool.rows(clean, b, n + M)
            for m in range(M):
                seen = tr.visible(n, M, m, window, sinks, *(masks[b] if masks else (None, None)))
                o, z, absv, peak, count = tr.attention(q[b, m].cpu().double().view(Hq, D), k, v, 0.125, seen)
                rel = ref.attention_tolerance(dtype, D, count, peak)[:, None]
                got = out[b, m].cpu().double().view(Hq, D)
                spoiled = torch.zeros(Hq, D, dtype=torch.bool)
                for (c, s, h), columns in bad.items():
                    if c == b and seen[s]:
                        spoiled[h * Hq // Hkv:(h + 1) * Hq // Hkv, list(columns)] = True
                assert torch.equal(~torch.isfinite(got), spoiled), (b, m, window)
                assert ((got - o).abs() <= U[dtype] * o.abs() + rel * absv + 1e-30)[~spoiled].all(), (b, m, window)
                assert ((lse[b, m].cpu().double() - z).abs() <= rel[:, 0] + 4 * U[F32] * (z.abs() + peak + 1)).all(), (b, m, window)
                spoiled_rows += int(spoiled.any())
        assert spoiled_rows


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,Hq", [(32, 2), (64, 4), (128, 16), (64, 32), (32, 64)])
@pytest.mark.parametrize("page", [16, 4])
def test_one_node_that_does_not_see_itself(dtype, D, Hq, page):
    """Any mask will do, one node's too: what lies in its own slot then has no influence."""
    lengths = [0, 1, 63, 64, 200]
    masks = [(np.zeros((1, 1), bool), np.zeros(1, np.int64))] * 5
    for value in (math.nan, math.inf):
        pool = Pool(5, 2, D, page, [n + 1 for n in lengths], dtype, seed=1)
        for b, n in enumerate(lengths):
            pool.put(pool.k, b, n, value)
            pool.put(pool.v, b, n, value)
        check(pool, dtype, Hq, 2, D, lengths, [1] * 5, 1, masks=masks)
        check(pool, dtype, Hq, 2, D, lengths, [1] * 5, 1, masks=masks, window=70, sinks=3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [9, 700])
def test_log_probabilities_of_large_logits(dtype, rows):
    """Logits far from 0: of the whole row, as tokens' marks, in front of or behind ordinary ones."""
    V = 6000
    g = torch.Generator().manual_seed(4)
    x = torch.randn(rows, V, generator=g)
    for r, big in enumerate((-1e9, -1e10, 3e9, 1e13, -7e20, 1e28)):
        x[r] = big * (1 + 1e-3 * x[r] if r % 2 else torch.ones(V))
    x[6, :5000] = -1e12
    x[7, 1000:] = -3e9
    x[8, ::2] = -1e29
    x = x.to(dtype).cuda()
    tokens = torch.randint(0, V, (rows, 2), generator=g, dtype=torch.int32).cuda()
    for scale in (1.0, 0.3, 40.0):
        check_logprobs(x[:9], V, scale, tokens[:9].contiguous(), 5)
    if rows > 9:
        check_logprobs(x, V, 1.0, tokens, 3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [6, 600])
def test_log_probabilities_at_scales_near_nothing(dtype, rows):
    """Tokens that cannot be stay so however small the scale is, and logits up to the type's largest count as what they are."""
    V = 3000
    g = torch.Generator().manual_seed(2)
    x = torch.randn(rows, V, generator=g)
    x[0, 100:] = -math.inf
    x[1, ::3] = -math.inf
    x[1] *= 1e29
    x[2] *= 1e38
    x[3] = torch.where(torch.arange(V) % 2 == 0, 3e38, -3e38)
    x[4, :7] = -2e30
    x[4, 7:] = -math.inf
    x[5] = torch.where(torch.arange(V) % 256 < 8, -9e29, -math.inf)
    x = x.to(dtype)
    x[torch.isinf(x) & (x > 0)] = torch.finfo(dtype).max
    tokens = torch.randint(0, V, (rows, 2), generator=g, dtype=torch.int32).cuda()
    x = x.cuda()
    for scale in (1e-26, 1e-28, 1e-30, 1e-34, 1e-37, 1e-38, 1e-40, 0.25, 1e-3):
        check_logprobs(x[:6], V, scale, tokens[:6].contiguous(), 5)
    if rows > 6:
        check_logprobs(x, V, 1e-30, tokens, 3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,Hq", [(3, 4), (40, 4), (70, 16)])
@pytest.mark.parametrize("score", [13.0, -13.0, 40.0])
def test_large_values_of_many_slots(dtype, M, Hq, score):
    """Scores that are alike, values near 2^112 (the sum of those of 8000 slots is below the largest fp32 number): their average is what comes out."""
    tsfm = lib()
    D, n = 64, 8000
    pool = Pool(2, 2, D, 16, [n + M, 100 + M], dtype, fill=0.0)
    pool.k[..., :] = 1.0
    pool.v[..., :] = 2.0 ** 112
    pool.v[..., 1::2] = -2.0 ** 112
    q = torch.full((2, M, Hq * D), score / D, device="cuda").to(dtype)
    out, lse = torch.zeros_like(q), torch.zeros(2, M, Hq, device="cuda")
    pages = pool.describe(tsfm)
    work = torch.empty(tsfm.tsfm_tree_attention_workspace(pages, 2, M, Hq, n + M), dtype=torch.uint8, device="cuda")
    mask, depth = tr.ancestors(tr.tree("random", M, 1))
    want = torch.full((D,), 2.0 ** 112, dtype=torch.float64, device="cuda")
    want[1::2] *= -1
    for tree in (True, False):
        args = (stream(), pages, q, q.stride(1), out, out.stride(1), ints([n, 100]), None)
        rest = (2, M, Hq, 1.0, 0, 0, n + M, lse, work, work.numel())
        if tree:
            tsfm.tsfm_tree_attention(*args, tr.words(mask).cuda(), ints(depth), True, *rest)
        else:
            tsfm.tsfm_window_attention(*args, *rest)
        # equal probabilities: their sum and the values' by the same rounded terms, up to n additions either way; one rounding of the result
        error = (out.double().view(2, M, Hq, D) / want - 1).abs().max()
        assert error <= 2 * (n + 300) * 2.0 ** -24 + {F32: 2.0 ** -24, BF16: 2.0 ** -8}[dtype], error


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [3, 600])
def test_log_probabilities_of_tokens_at_the_lowest_value(dtype, rows):
    """Finite, as their logits are."""
    V, low = 2000, torch.finfo(dtype).min
    x = torch.randn(rows, V, generator=torch.Generator().manual_seed(6)).to(dtype)
    x[0, ::2] = low
    x[1, 5:] = low
    x[2, 7] = -2.5e38
    tokens = torch.tensor([[4, 5, 7, 1999]] * rows, dtype=torch.int32).cuda()
    for scale in (1.0, 0.6):
        check_logprobs(x[:3].cuda(), V, scale, tokens[:3].contiguous(), 32)
    if rows > 3:
        check_logprobs(x.cuda(), V, 1.0, tokens, 2)
