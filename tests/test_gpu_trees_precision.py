"""bf16 attention of trees and windows with each of its outputs at the tolerance of its own type: the result is rounded once, log-sums never to bf16."""
import numpy as np
import pytest
import torch

from tests import serving_precision as sp
from tests import trees_precision as tp
from tests import trees_ref as tr
from tests.serving_ref import Pool
from tests.test_gpu_serving import BF16, ints, lib, stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("i", range(len(tp.CASES)))
@pytest.mark.parametrize("page", [16, 4])
def test_outputs_and_log_sums(i, page):
    tsfm = lib()
    given = tp.inputs(i)
    (D, Hq, Hkv, M, total, kind, window, sinks), length, masks, q, ks, vs = given
    B, longest, scale = len(total), max(total), D ** -0.5
    pool = Pool(B, Hkv, D, page, total, BF16, fill=0.0)
    for b, n in enumerate(total):
        s = torch.arange(n)
        at = pool.table[b].cpu()[s // page].long().cuda(), slice(None), (s % page).cuda()
        pool.k[at], pool.v[at] = ks[b].cuda(), vs[b].cuda()
    pages, qd = pool.describe(tsfm), q.cuda().view(B, M, Hq * D)
    out, lse = torch.zeros_like(qd), torch.zeros(B, M, Hq, device="cuda")
    work = torch.empty(tsfm.tsfm_tree_attention_workspace(pages, B, M, Hq, longest), dtype=torch.uint8, device="cuda")
    rest = (B, M, Hq, scale, window, sinks, longest, lse, work, work.numel())
    args = (stream(), pages, qd, Hq * D, out, Hq * D, ints(length), None)
    if masks is None:
        tsfm.tsfm_window_attention(*args, *rest)
    else:
        tsfm.tsfm_tree_attention(*args, torch.stack([tr.words(s) for s, _ in masks]).cuda(), ints(np.stack([d for _, d in masks])), False, *rest)
    out, lse = out.cpu().double().view(B, M, Hq, D), lse.cpu().double()
    worst = [0.0, 0.0]
    for b in range(B):
        for m in range(M):
            o, z, absv, peak, n = tp.exact(*given, b, m)
            worst[0] = max(worst[0], float(((out[b, m] - o).abs() / sp.out_tolerance(D, n, o, absv, peak)).max()))
            worst[1] = max(worst[1], float(((lse[b, m] - z).abs() / sp.lse_tolerance(D, n, z, peak)).max()))
    assert max(worst) <= 1.0, worst
