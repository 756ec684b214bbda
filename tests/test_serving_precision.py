"""The tolerances of tests/serving_precision.py tell two bf16 parts of a probability from one (host arithmetic, no GPU)."""
import pytest
import torch

from tests import serving_precision as sp


def with_parts(q, k, v, end, scale, parts):
    """Attention whose probabilities, relative to the largest, enter the product as so many bf16 parts; everything else in 64 bits, and the result
    rounded to bf16."""
    Hq, Hkv = q.shape[0], k.shape[1]
    kk, vv = (x[:end].double().repeat_interleave(Hq // Hkv, 1) for x in (k, v))
    s = torch.einsum("hd,nhd->hn", q.double(), kk) * scale
    p = torch.exp(s - s.amax(1, keepdim=True))
    used, rest = torch.zeros_like(p), p
    for _ in range(parts):
        part = rest.bfloat16().double()
        used, rest = used + part, rest - part
    return (torch.einsum("hn,nhd->hd", used, vv) / p.sum(1, keepdim=True)).bfloat16().double()


@pytest.mark.parametrize("i", range(len(sp.CASES)))
def test_one_part_fails_where_two_pass(i):
    D, Hq, Hkv, M, lengths = sp.CASES[i]
    lengths = [n + M - 1 for n in lengths]
    q, ks, vs = sp.inputs(D, Hq, Hkv, M, lengths, i)
    worst = {1: 0.0, 2: 0.0}
    for b, n in enumerate(lengths):
        for m in range(M):
            o, _, _, absv, peak, end, _ = sp.exact(q[b, m], ks[b], vs[b], n, M, m, D ** -0.5)
            tol = sp.out_tolerance(D, end, o, absv, peak)
            for parts in worst:
                worst[parts] = max(worst[parts], float(((with_parts(q[b, m], ks[b], vs[b], end, D ** -0.5, parts) - o).abs() / tol).max()))
    assert worst[2] <= 1.0 and worst[1] > 1.5, worst
