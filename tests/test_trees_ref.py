"""The reference of the trees' tests: its rule leaves the target's distribution, its masks are its parents' (no GPU needed)."""
import itertools

import numpy as np
import pytest

from tests import trees_ref as tr


def committed(p, q, children):
    """Distribution of the first committed token behind a root with `children` independent draws from q, by enumeration: the thresholds that
    tr.verify's rule gives each child, u uniform."""
    V, got = len(p), np.zeros(len(p))
    for xs in itertools.product(range(V), repeat=children):
        weight = np.prod([q[x] for x in xs])
        used, mass = 0.0, 1.0
        for x in xs:
            r = tr.rest(p, q, used, ())
            ok = min(1.0, r[x] / (q[x] * mass)) if q[x] * mass > 0 else 0.0
            got[x] += weight * ok
            weight *= 1 - ok
            used += mass
            mass = tr.rest(p, q, used, ()).sum()
        if weight > 0:
            r = tr.rest(p, q, used, ())
            r = r if r.sum() > 0 else p
            got += weight * r / r.sum()
    return got


@pytest.mark.parametrize("children", [1, 2, 3])
@pytest.mark.parametrize("seed", range(4))
def test_sampled_children_leave_the_targets_distribution(children, seed):
    rng = np.random.default_rng(seed)
    p, q = rng.dirichlet(np.ones(4) * 0.7, 2)
    # a few hundred terms of at most 1, each with a few roundings of 2^-53
    assert np.abs(committed(p, q, children) - p).max() < 1e-12


def test_picked_children_leave_the_targets_distribution():
    """Picks x_1, x_2 without a distribution: x_1 with p(x_1), x_2 with p(x_2) / (1 - p(x_1)) of what is left, else r."""
    p = np.array([0.5, 0.2, 0.2, 0.1])
    got, weight, mass, gone = np.zeros(4), 1.0, 1.0, set()
    for x in (2, 0):
        r = tr.rest(p, None, 0, gone)
        got[x] += weight * r[x] / mass
        weight *= 1 - r[x] / mass
        mass -= r[x]
        gone.add(x)
    r = tr.rest(p, None, 0, gone)
    got += weight * r / r.sum()
    assert np.abs(got - p).max() < 1e-12


def test_walks_end_where_the_rule_says():
    p = np.array([[0.0, 1.0, 0.0], [0.5, 0.5, 0.0], [1.0, 0.0, 0.0], [0.0, 0.0, 1.0]])
    # the root's first child (token 0) has no weight, its second (token 1) is taken, and that one's child (token 1) with u below 1/2
    tokens, parent = [9, 0, 1, 1], [-1, 0, 0, 2]
    p[2] = [0.5, 0.5, 0.0]
    assert tr.verify(tokens, parent, p, None, [0, 0.3, 0.9, 0.49, 0.1], 4) == ([1, 1, 2], [0, 2, 3])
    assert tr.verify(tokens, parent, p, None, [0, 0.3, 0.9, 0.51, 0.1], 4) == ([1, 0], [0, 2])
    assert tr.verify(tokens, parent, p, None, [0, 0.3, 0.9, 0.49, 0.1], 1) == ([1], [0])
    assert tr.verify(tokens, parent, p, None, [0.5] * 5, 0) == ([], [])


@pytest.mark.parametrize("kind", ["chain", "star", "binary", "random", "loose"])
def test_masks(kind):
    parent = tr.tree(kind, 70, 3)
    sees, depth = tr.ancestors(parent)
    for m in range(70):
        assert sees[m, m] and depth[m] == sees[m].sum() - 1 and not sees[m, m + 1:].any()
        if parent[m] >= 0:
            assert (sees[m] & ~sees[parent[m]]).sum() == 1 and depth[m] == depth[parent[m]] + 1
    bits = tr.words(sees)
    assert all(bool(int(bits[m, j // 64]) >> (j % 64) & 1) == sees[m, j] for m in range(70) for j in range(70))
    near, _ = tr.ancestors(parent, 2)
    assert (near.sum(1) == np.minimum(2, depth + 1)).all()
    if kind == "chain":                                        # a chain within a window is window attention
        for window, sinks in ((0, 0), (3, 0), (5, 2), (200, 9)):
            a, d = tr.ancestors(parent, window)
            for m in (0, 1, 7, 69):
                chain = tr.visible(20, 70, m, window, 0)
                assert (tr.visible(20, 70, m, window, 0, a, d) == chain).all()
                assert (tr.visible(20, 70, m, window, sinks)[:20] == tr.visible(20, 70, m, window, sinks, a, d)[:20]).all()
