"""Attention of trees and windows, log probabilities: batches, masks, values and scales that the ordinary cases (tests/test_gpu_trees.py) leave out."""
import pytest
import torch

from tests import trees_ref as tr
from tests.serving_ref import Pool
from tests.test_gpu_serving import stale
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
