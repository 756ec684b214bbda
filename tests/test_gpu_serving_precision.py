"""bf16 attention over pages with each of its outputs at the tolerance of its own type (tests/serving_precision.py): the result is rounded once, and
log-sums and weights are never rounded to bf16."""
import pytest
import torch

from tests import serving_precision as sp
from tests.serving_ref import Pool
from tests.test_gpu_serving import BF16, ints, lib, stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("i", range(len(sp.CASES)))
@pytest.mark.parametrize("page", [16, 4])
def test_outputs_log_sums_and_weights(i, page):
    tsfm = lib()
    D, Hq, Hkv, M, lengths = sp.CASES[i]
    lengths = [n + M - 1 for n in lengths]
    B, longest, scale = len(lengths), max(lengths), D ** -0.5
    q, ks, vs = sp.inputs(D, Hq, Hkv, M, lengths, i)
    pool = Pool(B, Hkv, D, page, lengths, BF16, fill=0.0)
    for b, n in enumerate(lengths):
        s = torch.arange(n)
        at = pool.table[b].cpu()[s // page].long().cuda(), slice(None), (s % page).cuda()
        pool.k[at], pool.v[at] = ks[b].cuda(), vs[b].cuda()
    pages, qd = pool.describe(tsfm), q.cuda().view(B, M, Hq * D)
    out, lse, w = torch.zeros_like(qd), torch.zeros(B, M, Hq, device="cuda"), torch.zeros(B, Hkv, longest, device="cuda")
    work = torch.empty(tsfm.tsfm_paged_attention_workspace(pages, B, M, Hq, longest, True), dtype=torch.uint8, device="cuda")
    tsfm.tsfm_paged_attention(stream(), pages, qd, Hq * D, out, Hq * D, ints([n - M for n in lengths]), None, B, M, Hq, scale, True, 0, longest, lse, None, w,
                              longest, work, work.numel())
    out, lse, w = out.cpu().double().view(B, M, Hq, D), lse.cpu().double(), w.cpu().double()
    worst = [0.0, 0.0, 0.0]
    for b, n in enumerate(lengths):
        want, allowed = torch.zeros(Hkv, n, dtype=torch.float64), torch.zeros(Hkv, n, dtype=torch.float64)
        for m in range(M):
            o, z, p, absv, peak, end, _ = sp.exact(q[b, m], ks[b], vs[b], n, M, m, scale)
            worst[0] = max(worst[0], float(((out[b, m] - o).abs() / sp.out_tolerance(D, end, o, absv, peak)).max()))
            worst[1] = max(worst[1], float(((lse[b, m] - z).abs() / sp.lse_tolerance(D, end, z, peak)).max()))
            want += p.view(Hkv, Hq // Hkv, n).sum(1)
            allowed += (p * sp.weight_tolerance(D, end, z, peak)[:, None]).view(Hkv, Hq // Hkv, n).sum(1)
        allowed += (M * Hq // Hkv + 1) * sp.U32 * want + 1e-30
        worst[2] = max(worst[2], float(((w[b, :, :n] - want).abs() / allowed).max()))
    assert max(worst) <= 1.0, worst
