"""Attention of trees and windows, log probabilities: batches, masks, values and scales that the ordinary cases (tests/test_gpu_trees.py) leave out."""
import pytest
import torch

from tests import trees_ref as tr
from tests.serving_ref import Pool
from tests.test_gpu_serving import ints, lib, stale, stream, wide
from tests.test_gpu_trees import BF16, check

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
