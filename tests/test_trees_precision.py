"""The tolerances tell two bf16 parts of a probability from one in the cases of tests/trees_precision.py (host arithmetic, no GPU)."""
import pytest

from tests import serving_precision as sp
from tests import trees_precision as tp


@pytest.mark.parametrize("i", range(len(tp.CASES)))
def test_one_part_fails_where_two_pass(i):
    given = tp.inputs(i)
    case = given[0]
    assert case[3] * case[1] // case[2] >= 17
    worst = {1: 0.0, 2: 0.0}
    for b in range(len(case[4])):
        for m in range(case[3]):
            o, _, absv, peak, n = tp.exact(*given, b, m)
            tol = sp.out_tolerance(case[0], n, o, absv, peak)
            for parts in worst:
                worst[parts] = max(worst[parts], float(((tp.with_parts(*given, b, m, parts) - o).abs() / tol).max()))
    assert worst[2] <= 1.0 and worst[1] > 1.5, worst
