"""bf16 attention of trees and windows with 17 rows of a key head and more, at the tolerances of tests/serving_precision.py: cases in which one rounding more
shows (probabilities that enter the product with the values as one bf16 part)."""
import numpy as np
import torch

from tests import serving_precision as sp
from tests import trees_ref as tr

# D, query heads, key heads, new tokens, slots of each series with them, tree or None (a chain), window, sinks
CASES = [(64, 20, 1, 1, [2, 12, 100], None, 0, 0), (128, 32, 1, 1, [40, 130], None, 64, 4), (128, 8, 1, 5, [7, 70, 130], "random", 0, 0),
         (64, 4, 2, 40, [64, 190], "random", 0, 0), (64, 8, 2, 70, [90, 300], "random", 60, 5), (128, 4, 2, 70, [80, 200], "binary", 0, 0),
         (128, 16, 1, 20, [50, 120], None, 30, 2), (64, 3, 1, 150, [200], None, 0, 0), (128, 5, 1, 60, [61, 150], "star", 0, 0)]


def inputs(i):
    """(case, length before the new tokens, masks or None, q, k and v of each series)"""
    D, Hq, Hkv, M, total, kind, window, sinks = CASES[i]
    q, ks, vs = sp.inputs(D, Hq, Hkv, M, total, i)
    return CASES[i], [n - M for n in total], None if kind is None else [tr.ancestors(tr.tree(kind, M, b)) for b in range(len(total))], q, ks, vs


def seen(case, length, masks, b, m):
    M, window, sinks = case[3], case[6], case[7]
    return tr.visible(length[b], M, m, window, sinks, *(masks[b] if masks else (None, None)))


def exact(case, length, masks, q, ks, vs, b, m):
    """(out, lse, the sum of p |v|, the largest sum of |q k| scale, slots)"""
    return tr.attention(q[b, m].double(), ks[b].double(), vs[b].double(), case[0] ** -0.5, seen(case, length, masks, b, m))


def with_parts(case, length, masks, q, ks, vs, b, m, parts):
    """As exact(), the probabilities relative to the largest so many bf16 parts, the result rounded to bf16."""
    D, Hq, Hkv = case[:3]
    idx = torch.from_numpy(np.flatnonzero(seen(case, length, masks, b, m)))
    kk, vv = (x[idx].double().repeat_interleave(Hq // Hkv, 1) for x in (ks[b], vs[b]))
    s = torch.einsum("hd,nhd->hn", q[b, m].double(), kk) * D ** -0.5
    p = torch.exp(s - s.amax(1, keepdim=True))
    used, rest = torch.zeros_like(p), p
    for _ in range(parts):
        part = rest.bfloat16().double()
        used, rest = used + part, rest - part
    return (torch.einsum("hn,nhd->hd", used, vv) / p.sum(1, keepdim=True)).bfloat16().double()
