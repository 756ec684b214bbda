"""Trees of drafted tokens, windows with sinks and log probabilities on the GPU against the definitions in 64 bits (tests/trees_ref.py)."""
import math

import numpy as np
import pytest
import torch

from tests import serving_ref as ref
from tests import trees_ref as tr
from tests.serving_ref import U, Pool
from tests.test_gpu_serving import ints, lib, make_rope, stale, stream, wide

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


# ------------------------------------------------------------------------------------------ masks
@pytest.mark.parametrize("M", [1, 2, 63, 64, 65, 200, 256])
def test_tree_init(M):
    tsfm = lib()
    kinds = ["chain", "star", "binary", "random", "loose", "random"]
    trees = [tr.tree(k, M, i) for i, k in enumerate(kinds)]
    trees[5][M - 1] = M                                        # not a node before it: counts as a root
    if M > 2:
        trees[5][2] = -9
    new = [M, M, max(0, M - 1), 0, M + 7, M]
    parent = ints(trees)
    for window in (0, 1, 3):
        mask = torch.full((6, M, (M + 63) // 64), -7, dtype=torch.int64, device="cuda")
        depth = torch.full((6, M), -7, dtype=torch.int32, device="cuda")
        tsfm.tsfm_tree_init(stream(), parent, ints(new), 6, M, window, mask, depth)
        for b in range(6):
            sees, d = tr.ancestors(trees[b], window)
            n = min(max(new[b], 0), M)
            sees[n:], d[n:] = False, 0
            assert torch.equal(mask[b].cpu(), tr.words(sees)) and depth[b].tolist() == d.tolist(), (b, window)
    one = torch.zeros(1, M, (M + 63) // 64, dtype=torch.int64, device="cuda")
    tsfm.tsfm_tree_init(stream(), parent[3:4], None, 1, M, 0, one, depth[:1])
    assert torch.equal(one[0].cpu(), tr.words(tr.ancestors(trees[3])[0]))


# ------------------------------------------------------------------------------------------ attention
def check(pool, dtype, Hq, Hkv, D, length, new, M, trees=None, shared=False, window=0, sinks=0, masks=None, qpad=0, seed=0, qfactor=2.0, scale=None,
          max_len=None, expect=None, runs=1, bad_rows=()):
    """trees: parents a series (one with shared), None: a chain; masks: (sees, depth) in their place.  bad_rows: (series, token) that may be anything not
    finite; expect: status."""
    tsfm = lib()
    B = pool.B
    new_cut = [min(max(n, 0), M) for n in new]
    total = [n + m for n, m in zip(length, new_cut)]
    max_len = max_len or max(1, max(total))
    scale = scale if scale is not None else 1 / math.sqrt(D)
    q = wide((B, M), Hq * D, dtype, qpad, seed + 1, qfactor)
    out = torch.full((B, M, Hq * D + qpad), -9.0, dtype=dtype, device="cuda")
    lse = torch.full((B, M, Hq), -9.0, device="cuda")
    pages = pool.describe(tsfm)
    size = tsfm.tsfm_tree_attention_workspace(pages, B, M, Hq, max_len)
    work = torch.full((size + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    if trees is not None:
        masks = [tr.ancestors(t) for t in trees]
    for _ in range(runs):
        if masks is None:
            tsfm.tsfm_window_attention(stream(), pages, q, q.stride(1), out, out.stride(1), ints(length), ints(new), B, M, Hq, scale, window, sinks, max_len,
                                       lse, work, size)
        else:
            bits, depth = torch.stack([tr.words(s) for s, _ in masks]).cuda(), ints(np.stack([d for _, d in masks]))
            tsfm.tsfm_tree_attention(stream(), pages, q, q.stride(1), out, out.stride(1), ints(length), ints(new), bits, depth, shared, B, M, Hq, scale,
                                     window, sinks, max_len, lse, work, size)
    torch.cuda.synchronize()
    assert int(pool.status) == (expect or 0)
    assert (work[size:] == 0xA5).all()
    got, z_got = out.cpu().double(), lse.cpu().double()
    assert (got[..., Hq * D:] == -9).all()
    for b in range(B):
        k, v = pool.rows(pool.k, b, total[b]), pool.rows(pool.v, b, total[b])
        for m in range(M):
            if m >= new_cut[b]:
                assert (got[b, m] == -9).all() and (z_got[b, m] == -9).all()
                continue
            mine = got[b, m, :Hq * D].view(Hq, D)
            if (b, m) in bad_rows:
                assert not torch.isfinite(mine).all()
                continue
            sees, depth = (None, None) if masks is None else masks[0 if shared else b]
            seen = tr.visible(length[b], new_cut[b], m, window, sinks, sees, depth)
            o, z, absv, peak, n = tr.attention(q[b, m].cpu().double().view(Hq, D), k, v, scale, seen)
            rel = ref.attention_tolerance(dtype, D, n, peak)[:, None]
            err = (mine - o).abs()
            assert (err <= U[dtype] * o.abs() + rel * absv + 1e-30).all(), (b, m, float(err.max()))
            if n:
                assert ((z_got[b, m] - z).abs() <= rel[:, 0] + 4 * U[F32] * (z.abs() + peak + 1)).all(), (b, m)
            else:
                assert (z_got[b, m] == -math.inf).all() and (mine == 0).all()
    return out, lse


LENGTHS = [0, 1, 5, 16, 60, 64, 65, 130, 200, 3, 513]
SHAPES = [(64, 8, 8, 7, 16, "heads"), (128, 32, 8, 9, 32, "slots"), (32, 4, 4, 5, 8, "heads"), (64, 20, 4, 26, 16, "heads"), (128, 6, 2, 33, 64, "slots"),
          (32, 12, 1, 3, 16, "slots"), (64, 3, 3, 70, 1, "heads"), (128, 7, 1, 17, 128, "heads"), (64, 16, 1, 1, 32, "slots"), (128, 2, 1, 1, 8, "slots"),
          (64, 2, 1, 130, 16, "heads"), (128, 16, 2, 65, 16, "heads"), (64, 5, 1, 40, 4, "slots"), (128, 3, 3, 2, 16, "heads"), (32, 6, 3, 90, 16, "heads")]


def new_of(M, B):
    return [M if i % 3 != 2 else (M * i) // B for i in range(B)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,Hq,Hkv,M,page,order", SHAPES)
@pytest.mark.parametrize("window,sinks,shared", [(0, 0, False), (37, 3, True), (4, 70, False)])
def test_tree_attention(dtype, D, Hq, Hkv, M, page, order, window, sinks, shared):
    B = len(LENGTHS)
    new = new_of(M, B)
    pool = Pool(B, Hkv, D, page, [n + m for n, m in zip(LENGTHS, new)], dtype, order, seed=D + M)
    kinds = ["random", "chain", "star", "binary", "loose"]
    trees = [tr.tree(kinds[(b + M) % 5], M, b) for b in range(1 if shared else B)]
    for b in range(B):
        stale(pool, b, LENGTHS[b] + new[b])
    check(pool, dtype, Hq, Hkv, D, LENGTHS, new, M, trees, shared, window, sinks, qpad=16 if M % 2 else 0, seed=M)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,Hq,Hkv,M,page,order", SHAPES + [(128, 8, 2, 300, 16, "heads"), (64, 4, 4, 200, 64, "slots"), (64, 12, 4, 150, 2, "heads")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (50, 4), (200, 65), (5, 600)])
def test_window_attention(dtype, D, Hq, Hkv, M, page, order, window, sinks):
    lengths = LENGTHS if M < 100 else [0, 1, 64, 250]
    B = len(lengths)
    new = new_of(M, B)
    pool = Pool(B, Hkv, D, page, [n + m for n, m in zip(lengths, new)], dtype, order, seed=D + M)
    for b in range(B):
        stale(pool, b, lengths[b] + new[b])
    check(pool, dtype, Hq, Hkv, D, lengths, new, M, None, False, window, sinks, seed=M)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,Hq,D", [(6, 4, 64), (24, 8, 128), (70, 8, 64)])
def test_any_mask_and_rows_that_see_nothing(dtype, M, Hq, D):
    """Masks of no tree (later tokens, not oneself, nothing), the cache empty or hidden by the window."""
    rng = np.random.default_rng(M)
    lengths = [0, 0, 70, 200]
    masks = []
    for b in range(4):
        sees = rng.random((M, M)) < [0.3, 0.0, 0.5, 0.02][b]
        sees[::3] = False
        masks.append((sees, rng.integers(0, M, M)))
    pool = Pool(4, 2, D, 16, [n + M for n in lengths], dtype, seed=1)
    check(pool, dtype, Hq, 2, D, lengths, [M] * 4, M, masks=masks)
    check(pool, dtype, Hq, 2, D, lengths, [M, M, M - 1, M], M, masks=masks, window=1)        # nothing of the cache, but for the root's depth 0: slot len - 0 .. none
    check(pool, dtype, Hq, 2, D, lengths, [M] * 4, M, masks=masks, window=2, sinks=1)


def test_series_without_tokens_and_lengths_outside_the_capacity():
    tsfm = lib()
    for M, new in ((5, [0, 0, 0]), (5, [-3, 5, 9]), (40, [0, 40, 1])):
        pool = Pool(3, 2, 64, 16, [60, 60, 80], BF16, seed=M)
        check(pool, BF16, 16, 2, 64, [10, 20, 33], new, M, [tr.tree("random", M, b) for b in range(3)])
        check(pool, BF16, 16, 2, 64, [10, 20, 33], new, M, None, window=7, sinks=2)
    # a negative length counts as 0, one beyond the capacity is cut to it; both are reported
    pool = Pool(2, 2, 64, 16, [64, 64], BF16, seed=2)
    q = wide((2, 3), 4 * 64, BF16, 0, 1)
    out, ws = torch.zeros_like(q), torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    tsfm.tsfm_window_attention(stream(), pool.describe(tsfm), q, q.stride(1), out, out.stride(1), ints([-5, 1000]), None, 2, 3, 4, 0.125, 8, 2, 64, None, ws,
                               ws.numel())
    torch.cuda.synchronize()
    assert int(pool.status) & tsfm.TSFM_PAGES_BAD_LEN and torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,Hq", [(9, 2), (26, 4), (80, 8)])
def test_values_that_are_not_finite_reach_only_tokens_that_see_them(dtype, M, Hq):
    D, lengths, window, sinks = 64, [150, 40], 30, 4
    parent = [tr.tree("random", M, 5), tr.tree("star", M, 0)]
    pool = Pool(2, 2, D, 16, [n + M for n in lengths], dtype, seed=3)
    bad = {(0, 10), (0, 125), (0, 150 + 3), (1, 40 + 5)}       # hidden to all; in some windows; two nodes
    for b, s in bad:
        pool.put(pool.k, b, s, math.nan)
        pool.put(pool.v, b, s, math.inf if s % 2 else math.nan)
    for masks in ([tr.ancestors(p) for p in parent], None):
        hit = set()
        for b in range(2):
            for m in range(M):
                seen = tr.visible(lengths[b], M, m, window, sinks, *(masks[b] if masks else (None, None)))
                if any(seen[s] for c, s in bad if c == b):
                    hit.add((b, m))
        assert hit and len(hit) < 2 * M
        check(pool, dtype, Hq, 2, D, lengths, [M, M], M, masks=masks, window=window, sinks=sinks, bad_rows=hit)


@pytest.mark.parametrize("M", [3, 40])
def test_pages_outside_the_pool_are_not_followed(M):
    tsfm = lib()
    pool = Pool(2, 2, 64, 16, [100 + M, 100 + M], BF16, seed=4)
    pool.table[0, 2], pool.table[1, 0] = 10 ** 6, -3
    q = wide((2, M), 4 * 64, BF16, 0, 1)
    out, ws = torch.zeros_like(q), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    tsfm.tsfm_window_attention(stream(), pool.describe(tsfm), q, q.stride(1), out, out.stride(1), ints([100, 100]), None, 2, M, 4, 0.125, 0, 0, 100 + M, None,
                               ws, ws.numel())
    torch.cuda.synchronize()
    assert int(pool.status) == tsfm.TSFM_PAGES_BAD_ID and torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_caches_are_shared_by_ctas(dtype):
    """One series over many CTAs, and the same answer twice."""
    for M, Hq, window in ((1, 8, 0), (12, 8, 0), (40, 8, 9000), (1, 8, 5000)):
        pool = Pool(1, 2, 64, 64, [20000 + M], dtype, seed=5)
        a = check(pool, dtype, Hq, 2, 64, [20000], [M], M, [tr.tree("random", M, 1)] if M > 1 else None, window=window, sinks=70 if window else 0)
        b = check(pool, dtype, Hq, 2, 64, [20000], [M], M, [tr.tree("random", M, 1)] if M > 1 else None, window=window, sinks=70 if window else 0, runs=2)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_window_without_bound_is_paged_attention():
    tsfm = lib()
    for M in (1, 9, 50):
        lengths = [0, 100, 300]
        pool = Pool(3, 2, 64, 16, [n + M for n in lengths], BF16, seed=6)
        q = wide((3, M), 8 * 64, BF16, 0, 1)
        a, b, ws = torch.zeros_like(q), torch.zeros_like(q), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
        pages, n = pool.describe(tsfm), ints(lengths)
        tsfm.tsfm_window_attention(stream(), pages, q, q.stride(1), a, a.stride(1), n, None, 3, M, 8, 0.125, 0, 0, 300 + M, None, ws, ws.numel())
        tsfm.tsfm_paged_attention(stream(), pages, q, q.stride(1), b, b.stride(1), n, None, 3, M, 8, 0.125, True, 0, 300 + M, None, None, None, 0, ws,
                                  ws.numel())
        # each within a rounding to bf16, and of the probabilities, of the exact result: |v| is below 5 here
        assert (a.double() - b.double()).abs().max() <= 4 * 2.0 ** -8 * 5


# ------------------------------------------------------------------------------------------ append at depths
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout,rot", [("half", 64), ("interleaved", 32), ("half", 6)])
@pytest.mark.parametrize("shared", [False, True])
def test_rope_append_tree_is_append_at_each_nodes_position(dtype, layout, rot, shared):
    tsfm = lib()
    B, M, Hq, Hkv, D = 3, 21, 6, 2, 64
    depth = np.stack([tr.ancestors(tr.tree("random", M, b))[1] for b in range(1 if shared else B)])
    length, pos, new = [3, 40, 100], [7, 5000, 2 ** 30], [M, 4, M]
    rope, _ = make_rope(layout, rot, "plain")
    qkv = wide((B, M), (Hq + 2 * Hkv) * D, dtype, 0, 1)
    got, want = (Pool(B, Hkv, D, 16, [n + M for n in length], dtype, seed=1, fill=0.0) for _ in range(2))
    q_got, q_want = (torch.zeros(B, M, Hq * D, dtype=dtype, device="cuda") for _ in range(2))
    tsfm.tsfm_rope_append_tree(stream(), rope, got.describe(tsfm), qkv, qkv.stride(1), q_got, q_got.stride(1), ints(pos), ints(length), ints(new), ints(depth),
                               shared, B, M, Hq)
    for m in range(M):                                         # token by token, its position given
        d = depth[:, m] if not shared else depth[:, m].repeat(B)
        x, y = qkv[:, m:m + 1].contiguous(), torch.zeros(B, 1, Hq * D, dtype=dtype, device="cuda")
        tsfm.tsfm_rope_append(stream(), rope, want.describe(tsfm), x, x.stride(1), y, y.stride(1), ints([p + int(e) for p, e in zip(pos, d)]),
                              ints([n + m for n in length]), ints([int(m < n) for n in new]), B, 1, Hq)
        q_want[:, m] = y[:, 0]
    assert torch.equal(q_got, q_want) and torch.equal(got.k, want.k) and torch.equal(got.v, want.v)


# ------------------------------------------------------------------------------------------ log probabilities
def check_logprobs(x, V, scale, tokens, n_top, names=("lse", "entropy")):
    """x: [rows, >= V] on the GPU (a view at any offset)."""
    tsfm = lib()
    rows, n_tok = x.shape[0], tokens.shape[1] if tokens is not None else 0
    logprob = torch.full((rows, n_tok), 7.0, device="cuda") if n_tok else None
    lse, entropy = (torch.full((rows,), 7.0, device="cuda") if n in names else None for n in ("lse", "entropy"))
    ids, best = (torch.full((rows, n_top), -5, dtype=torch.int32, device="cuda"), torch.full((rows, n_top), 7.0, device="cuda")) if n_top else (None, None)
    tsfm.tsfm_token_logprobs(stream(), x, x.stride(0), rows, V, scale, tokens, n_tok, logprob, lse, entropy, n_top, ids, best)
    torch.cuda.synchronize()
    s32 = float(np.float32(scale))
    for r in range(rows):
        raw = x[r, :V].cpu()
        lp, z, h, want_ids, want_best = tr.logprobs(raw.float(), s32, tokens[r].tolist() if n_tok else [], n_top)
        if n_top:
            assert ids[r].tolist() == want_ids, r
        live = raw.float()[torch.isfinite(raw.float())].double() * s32
        high = float(live.max()) if len(live) else 0.0
        # an exponent x scale - max scale in base 2: three roundings of numbers of at most 1.45 (|x| + |max|) scale, of which only those
        # within 300 of the maximum count; the exponential 2^-22; sums of V terms in some order, a few hundred in a row and a tree
        u = 2.0 ** -24
        span = 1.45 * (2 * abs(high) + 210)
        steps = V / 256 + 64
        tol = 3 * u * span + 2.0 ** -22 + steps * u

        def close(got, exact, more):
            if math.isnan(exact) or math.isinf(exact):
                assert (math.isnan(got) if math.isnan(exact) else got == exact), (r, got, exact)
            else:
                assert abs(got - exact) <= tol + more, (r, got, exact)

        if lse is not None:
            close(float(lse[r]), z, 3 * u * (abs(z) if math.isfinite(z) else 0))
        if entropy is not None:                                # sums of p d, |d| up to log V where it counts: relative to 1 + that
            close(float(entropy[r]), h, (tol + 4 * u) * (2 + 2 * math.log(V + 1)))
        for got, exact in zip(logprob[r].tolist() if n_tok else [], lp):
            close(got, exact, 4 * u * (abs(exact) if math.isfinite(exact) else 0))
        for got, exact in zip(best[r].tolist() if n_top else [], want_best):
            close(got, exact, 4 * u * (abs(exact) if math.isfinite(exact) else 0))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,rows,pad,offset", [(1, 3, 0, 0), (2, 5, 1, 0), (7, 4, 0, 3), (31, 9, 2, 1), (255, 7, 0, 5), (1000, 300, 0, 0), (1025, 5, 7, 0),
                                               (4096, 2, 0, 0), (8193, 700, 0, 1), (32003, 1, 0, 0), (50001, 3, 5, 7), (131072, 2, 0, 0)])
def test_token_logprobs(dtype, V, rows, pad, offset):
    g = torch.Generator().manual_seed(V)
    flat = (torch.randn(rows * (V + pad) + offset, generator=g) * 3).to(dtype).cuda()
    x = flat[offset:].view(rows, V + pad)
    for n_tok, n_top, scale in ((1, 5, 1.0), (0, 0, 0.7), (3, 32, 1.7)):
        tokens = torch.randint(0, V, (rows, n_tok), generator=g, dtype=torch.int32).cuda() if n_tok else None
        if n_tok == 3:
            tokens[0, 1], tokens[-1, 0] = -1, V                # no tokens
        check_logprobs(x if rows < 100 else x[:40], V, scale, tokens if rows < 100 or tokens is None else tokens[:40].contiguous(), n_top)
    if rows >= 100:                                            # many rows: a CTA a row
        check_logprobs(x, V, 1.0, None, 3)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs_of_odd_rows(dtype):
    V = 5000
    g = torch.Generator().manual_seed(1)
    x = torch.randn(14, V, generator=g) * 2
    x[0] = -math.inf
    x[1] = 0.25                                                # all equal: the lowest tokens
    x[2, :] = -math.inf
    x[2, 4321] = 1.0                                           # one token left
    x[3, 7::9] = -math.inf
    x[4, 100] = math.nan
    x[5, 100] = math.inf
    x[6] = torch.arange(V) / 64.0                              # ascending: the best lie together at the end
    x[7] = -torch.arange(V) / 64.0
    x[8] = math.nan
    x[9, :] = torch.finfo(dtype).min
    x[10] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)
    x[11, 1000:1700] = 50.0 + torch.arange(700) / 1e3          # hundreds above the rest
    x[12] *= 1e4
    x[13, :] = -1e30
    x[13, 5] = 80.0
    tokens = torch.tensor([[0, 4321, 1005]] * 14, dtype=torch.int32).cuda()
    for C_rows in (14, 1):                                     # one CTA a row, and rows shared by CTAs
        for r in range(0, 14, C_rows):
            check_logprobs(x[r:r + C_rows].to(dtype).cuda(), V, 1.0, tokens[r:r + C_rows].contiguous(), 20)
    # a period of the threads' columns: everything large lies in few of them
    y = torch.zeros(1, 200000)
    for p in (2048, 1024, 256):
        y[0, ::p] = 1.0 + torch.arange(len(y[0, ::p])) / 1e4
    check_logprobs(y.to(dtype).cuda(), 200000, 1.0, None, 32)
    many = y.expand(600, -1).to(dtype).cuda()
    check_logprobs(many[:, :150000], 150000, 1.0, None, 4, names=())


# ------------------------------------------------------------------------------------------ verification of a tree
def run_verify(tokens, parent, p, q, u, new, length, shared=False, seed=0, rnd=0, s0=0):
    tsfm = lib()
    B, M, V = p.shape
    out, path = (torch.full((B, M), -5, dtype=torch.int32, device="cuda") for _ in range(2))
    n, len_out = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    tsfm.tsfm_verify_tree(stream(), tokens, parent, shared, p, p.stride(1), q, q.stride(1) if q is not None else 0, B, M, V, u, seed, rnd, s0, new, length, out,
                          path, n, len_out if length is not None else None)
    torch.cuda.synchronize()
    return out.cpu(), path.cpu(), n.cpu(), len_out.cpu()


def check_verify(tokens, parent, p, q, u, new, shared=False):
    B, M, V = p.shape
    length = torch.arange(B, dtype=torch.int32, device="cuda") * 10
    out, path, n, len_out = run_verify(tokens, parent, p, q, u, new, length, shared)
    deepest = 0
    for b in range(B):
        nodes = M if new is None else min(max(int(new[b]), 0), M)
        w = lambda x: ref.weight(x[b].cpu().numpy())
        want, way = tr.verify(tokens[b].tolist(), parent[0 if shared else b].tolist(), w(p), None if q is None else w(q), u[b].tolist(), nodes)
        assert path[b].tolist() == way + [-1] * (M - len(way)), b
        assert out[b].tolist() == want + [-1] * (M - len(want)), b
        assert int(n[b]) == max(0, len(way) - 1) and int(len_out[b]) == 10 * b + len(way)
        deepest = max(deepest, len(way))
    return deepest


def drafted(B, M, V, seed, sampled, kind="random", noise=0.5):
    g = torch.Generator().manual_seed(seed)
    trees = torch.tensor([tr.tree(kind, M, seed + b) for b in range(B)], dtype=torch.int32)
    x = torch.randn(B, M, V, generator=g) * 2
    q = torch.softmax(x, -1)
    p = torch.softmax(x + noise * torch.randn(x.shape, generator=g), -1)
    tokens = torch.zeros(B, M, dtype=torch.int32)
    for b in range(B):
        count = {}
        for m in range(1, M):
            up = max(0, int(trees[b, m]))
            if sampled:
                tokens[b, m] = torch.multinomial(q[b, up], 1, generator=g)[0]
            else:
                i = count.get(up, 0)
                tokens[b, m] = q[b, up].argsort(descending=True)[min(i, V - 1)]
                count[up] = i + 1
    u = torch.rand(B, M + 1, generator=g)
    return tokens.cuda(), trees.cuda(), p.cuda(), q.cuda() if sampled else None, u.cuda()


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("B,M,V", [(1, 1, 5), (1, 8, 32003), (9, 33, 100), (40, 16, 1000), (3, 70, 257), (2, 256, 40), (300, 7, 300), (5, 12, 70001)])
def test_verify_tree(sampled, B, M, V):
    deepest = 0
    for seed, kind, noise in ((0, "random", 0.4), (1, "star", 1.5), (2, "chain", 0.2), (3, "loose", 0.7)):
        t, tree, p, q, u = drafted(B, M, V, seed, sampled, kind, noise)
        new = None if seed == 0 else ints([max(0, M - (b * 3) % (M + 2)) for b in range(B)])
        deepest = max(deepest, check_verify(t, tree, p, q, u, new))
        if seed == 1:
            check_verify(t, tree[:1].contiguous(), p, q, u, new, shared=True)
        if V * B * M > 3e6:
            break
    assert deepest > 1 or M == 1 or (not sampled and V > 1000)        # (of a large vocabulary even the best tokens are seldom drawn)


def test_verify_tree_edges():
    """Entries that are no probabilities, tokens outside the vocabulary, the same child twice, a target that equals the draft, rows without weight."""
    B, M, V = 12, 9, 333
    for sampled in (True, False):
        t, tree, p, q, u = drafted(B, M, V, 7, sampled, "star", 0.8)
        t[1, 1:] = ints([-1, V, 2 ** 31 - 1, -2 ** 31] * 2)
        t[2, 2:] = t[2, 1].clone()
        p[3, 0] = 0
        p[4, 0, ::2] = -1.0
        p[4, 0, 1] = math.nan
        p[5, 0, 5] = math.inf
        if sampled:
            q[6] = p[6]
            q[7, 0] = 0
            q[8, 0, ::3] = math.nan
            q[9, 0] = p[9, 0] * 3                              # nothing is left after a rejection
        u[10] = ints([0] * (M + 1)).float()
        u[11] = 1.0
        u[9] = math.nan if not sampled else 0.9999
        check_verify(t, tree, p, q, u, None)
        tree[0, 3] = 3                                         # its own parent: no node leads there
        tree[0, 4] = 8
        check_verify(t, tree, p, q, u, ints([M] * B))


def test_verify_tree_of_a_chain_is_verify_tokens():
    tsfm = lib()
    B, K, V = 20, 6, 500
    t, tree, p, q, u = drafted(B, K + 1, V, 11, True, "chain", 0.4)
    out, path, n, _ = run_verify(t, tree, p, q, u, None, None)
    # proposal i of the chain is node i + 1: its uniform there, its row of q at node i
    a, na = torch.zeros(B, K + 1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    qs = q[:, :K].contiguous()
    tsfm.tsfm_verify_tokens(stream(), t[:, 1:].contiguous(), p, V, qs, V, B, K, V, u[:, 1:].contiguous(), 0, 0, 0, None, None, a, na, None)
    assert torch.equal(out, a.cpu()) and torch.equal(n, na.cpu())
    for b in range(B):
        assert path[b].tolist() == list(range(int(n[b]) + 1)) + [-1] * (K - int(n[b]))


def test_verify_tree_with_the_librarys_uniforms():
    from oracle import tsfm_oracle as orc
    B, M, V = 6, 11, 77
    t, tree, p, q, _ = drafted(B, M, V, 5, True)
    u = torch.tensor([[orc.acceptance_uniform(0x123456789, 4 + b, 9, i) for i in range(M + 1)] for b in range(B)], dtype=torch.float32).cuda()
    a = run_verify(t, tree, p, q, None, None, None, seed=0x123456789, rnd=9, s0=4)
    again = run_verify(t, tree, p, q, None, None, None, seed=0x123456789, rnd=9, s0=4)
    assert all(torch.equal(x, y) for x, y in zip(a, again))
    b = run_verify(t, tree, p, q, u, None, None)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


# ------------------------------------------------------------------------------------------ commit
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,Hkv,page,order,layers,M", [(64, 3, 16, "heads", 1, 20), (128, 8, 8, "slots", 3, 61), (32, 1, 1, "heads", 5, 256), (128, 1, 64, "heads", 2, 1)])
def test_cache_commit(dtype, D, Hkv, page, order, layers, M):
    tsfm = lib()
    rng = np.random.default_rng(M)
    lengths = [0, 5, 16, 100, 7, 33, 64, 1]
    B = len(lengths)
    pool = Pool(B, Hkv, D, page, [n + M for n in lengths], dtype, order, seed=2)
    k, v = (torch.randn(layers, *x.shape, generator=torch.Generator().manual_seed(i)).to(dtype).cuda() for i, x in enumerate((pool.k, pool.v)))
    if order == "slots":
        k, v = (x.transpose(2, 3).contiguous().transpose(2, 3) for x in (k, v))
    paths = np.full((B, M), -1, np.int64)
    for b in range(B):
        n = min(M, [1, 2, M, (M + 1) // 2, 9, M, 0, 1][b])
        paths[b, :n] = np.sort(rng.choice(M, n, replace=False)) if b in (1, 3, 4) else np.arange(n)
    paths[7, :1] = M - 1
    if M > 10:
        paths[5, 4:8] = [6, 6, 8, 9]                           # ends at the second 6
    want_k, want_v = k.cpu().clone(), v.cpu().clone()
    table = pool.table.cpu().long()
    for b in range(B):
        last = -1
        for i, s in enumerate(paths[b]):
            if s <= last or s >= M:
                break
            last = s
            a, c = lengths[b] + int(s), lengths[b] + i
            for x in (want_k, want_v):
                x[:, table[b, c // page], :, c % page] = x[:, table[b, a // page], :, a % page]
    pages = tsfm.kv_pages(k[0], v[0], pool.table, pool.status)
    tsfm.tsfm_cache_commit(stream(), pages, ints(paths), ints(lengths), B, M, layers, k.stride(0))
    torch.cuda.synchronize()
    assert torch.equal(k.cpu(), want_k) and torch.equal(v.cpu(), want_v) and int(pool.status) == 0


def test_commits_outside_the_pool_are_left_alone():
    tsfm = lib()
    pool = Pool(3, 2, 64, 16, [64] * 3, BF16, seed=2)
    pool.table[0, 1] = 999
    before = pool.k.clone(), pool.v.clone()
    path = ints([[0, 20], [0, 20], [0, 20]])
    pages = pool.describe(tsfm)
    tsfm.tsfm_cache_commit(stream(), pages, path, ints([0, 0, 0]), 1, 2)               # M 2: node 20 is none
    assert int(pool.status) == 0
    path = torch.full((3, 40), -1, dtype=torch.int32, device="cuda")
    path[:, 0], path[:, 1] = 0, 30
    tsfm.tsfm_cache_commit(stream(), pages, path, ints([0, 50, -2]), 3, 40)
    torch.cuda.synchronize()
    assert int(pool.status) == tsfm.TSFM_PAGES_BAD_ID | tsfm.TSFM_PAGES_BAD_LEN
    # series 0: slot 30 lies in a page outside the pool; series 1: slot 80 behind the capacity; series 2: slots -2 and -1
    assert torch.equal(pool.k, before[0]) and torch.equal(pool.v, before[1])


# ------------------------------------------------------------------------------------------ together
def rounds(seed, graph=False):
    """Rounds of a model over a cache of pages: a tree is appended, attended to, verified, its path committed.  Yields after each round."""
    tsfm = lib()
    B, M, Hq, Hkv, D, V, page, layers = 4, 23, 8, 2, 64, 200, 16, 2
    g = torch.Generator().manual_seed(seed)
    length = [0, 30, 64, 100]
    shape = (layers, B * 20, Hkv, page, D)
    k, v = (torch.zeros(shape, dtype=BF16, device="cuda") for _ in "kv")
    table = torch.randperm(B * 20, generator=g).view(B, 20).int().cuda()
    pages = [tsfm.kv_pages(k[i], v[i], table) for i in range(layers)]
    rope, f = make_rope("half", D, "plain")
    lens = ints(length)
    # keys and values of what is there already
    old = torch.randn(layers, B, 100, (Hq + 2 * Hkv) * D, generator=g).to(BF16).cuda()
    for i in range(layers):
        tsfm.tsfm_rope_append(stream(), rope, pages[i], old[i], old[i].stride(1), None, 0, None, ints([0] * B), lens, B, 100, Hq)
    history = [[old[:, b, n].cpu() for n in range(length[b])] for b in range(B)]
    size = tsfm.tsfm_tree_attention_workspace(pages[0], B, M, Hq, 320)
    work = torch.empty(size, dtype=torch.uint8, device="cuda")
    mask, depth = torch.zeros(B, M, 1, dtype=torch.int64, device="cuda"), torch.zeros(B, M, dtype=torch.int32, device="cuda")
    parent, tokens = torch.zeros(B, M, dtype=torch.int32, device="cuda"), torch.zeros(B, M, dtype=torch.int32, device="cuda")
    qkv, out = torch.zeros(layers, B, M, (Hq + 2 * Hkv) * D, dtype=BF16, device="cuda"), torch.zeros(layers, B, M, Hq * D, dtype=BF16, device="cuda")
    q = torch.zeros(B, M, Hq * D, dtype=BF16, device="cuda")
    p, dist, u = torch.zeros(B, M, V, device="cuda"), torch.zeros(B, M, V, device="cuda"), torch.zeros(B, M + 1, device="cuda")
    drawn, path = (torch.zeros(B, M, dtype=torch.int32, device="cuda") for _ in range(2))
    n, len_out = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")

    def step():
        s = stream()
        tsfm.tsfm_tree_init(s, parent, None, B, M, 0, mask, depth)
        for i in range(layers):
            tsfm.tsfm_rope_append_tree(s, rope, pages[i], qkv[i], qkv[i].stride(1), q, q.stride(1), None, lens, None, depth, False, B, M, Hq)
            tsfm.tsfm_tree_attention(s, pages[i], q, q.stride(1), out[i], out[i].stride(1), lens, None, mask, depth, False, B, M, Hq, 0.125, 0, 0, 320, None,
                                     work, size)
        tsfm.tsfm_verify_tree(s, tokens, parent, False, p, V, dist, V, B, M, V, u, 0, 0, 0, None, lens, drawn, path, n, len_out)
        tsfm.tsfm_cache_commit(s, pages[0], path, lens, B, M, layers, k.stride(0))
        lens.copy_(len_out)

    captured = None
    for r in range(4):
        t, tr_, pp, qq, uu = drafted(B, M, V, 100 * seed + r, True, "random", 0.5)
        for dst, src in ((tokens, t), (parent, tr_), (p, pp), (dist, qq), (u, uu), (qkv, torch.randn(qkv.shape, generator=g).to(BF16).cuda())):
            dst.copy_(src)
        if graph and captured is None:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured, stream=side):
                step()
        if graph:
            captured.replay()
        else:
            step()
        torch.cuda.synchronize()
        yield dict(B=B, M=M, Hq=Hq, Hkv=Hkv, D=D, page=page, layers=layers, k=k, v=v, table=table, f=f, history=history, qkv=qkv, out=out, path=path, n=n,
                   lens=lens, parent=parent, drawn=drawn)


@pytest.mark.parametrize("graph", [False, True])
def test_rounds_of_a_served_model_with_trees(graph):
    """Each node's attention is that of a chain that holds its ancestors alone, and after the commit the cache is as if only the accepted tokens had ever
    been appended."""
    for state in rounds(3, graph):
        s = state
        B, M, Hq, Hkv, D = (s[x] for x in ("B", "M", "Hq", "Hkv", "D"))
        for b in range(B):
            past, way = s["history"][b], [x for x in s["path"][b].tolist() if x >= 0]
            sees, depth = tr.ancestors(s["parent"][b].tolist())
            for layer in range(s["layers"]):
                row = lambda x, t: ref.turn(x[layer].double().view(-1, D)[:Hq + Hkv], t, s["f"], "half").to(BF16).double()
                old = [row(x, t) for t, x in enumerate(past)]
                new = [row(s["qkv"][:, b, m].cpu(), len(past) + int(depth[m])) for m in range(M)]
                values = [x[layer].double().view(-1, D)[Hq + Hkv:] for x in past] + [s["qkv"][layer, b, m].cpu().double().view(-1, D)[Hq + Hkv:] for m in range(M)]
                keys = [x[Hq:] for x in old + new]
                kk, vv = torch.stack(keys), torch.stack(values)
                for m in (0, M // 2, M - 1, way[-1]):
                    seen = tr.visible(len(past), M, m, 0, 0, sees, depth)
                    o, _, absv, peak, n = tr.attention(new[m][:Hq], kk, vv, 0.125, seen)
                    # beside the attention's own: queries and keys that were rounded to bf16 on one side of a border here, on the other there, a
                    # step of 2^-7 of an element in some products: 2^-6 of the score's peak at the very most
                    rel = ref.attention_tolerance(BF16, D, n, peak)[:, None] + 2 * 2.0 ** -6 * peak[:, None]
                    assert ((s["out"][layer, b, m].cpu().double().view(Hq, D) - o).abs() <= U[BF16] * o.abs() + rel * absv).all(), (b, layer, m)
            past += [s["qkv"][:, b, m].cpu().clone() for m in way]
            assert int(s["lens"][b]) == len(past) and int(s["n"][b]) == len(way) - 1
            t = s["table"][b].cpu().long()
            for layer in range(s["layers"]):
                for i, x in enumerate(past):
                    at = (layer, t[i // s["page"]], slice(None), i % s["page"])
                    z = x[layer].double().view(-1, D)
                    want = ref.turn(z[:Hq + Hkv], float(i), s["f"], "half")[Hq:]
                    assert torch.equal(s["v"].cpu()[at].double(), z[Hq + Hkv:])
                    assert ((s["k"].cpu()[at].double() - want).abs() <= U[BF16] * want.abs() + 2.0 ** -20 * z.abs().max()).all()


def test_calls_on_two_streams_at_once():
    """Each with a workspace of its own; the same results as one after the other."""
    tsfm = lib()
    M, lengths = 40, [2000, 900, 50]
    pool = Pool(3, 4, 128, 32, [n + M for n in lengths], BF16, seed=7)
    pages = pool.describe(tsfm)
    mask, depth = tr.ancestors(tr.tree("random", M, 1))
    mask, depth = tr.words(mask).cuda(), ints(depth)
    q = [wide((3, M), 16 * 128, BF16, 0, i) for i in range(2)]
    out = [torch.zeros_like(x) for x in q]
    size = tsfm.tsfm_tree_attention_workspace(pages, 3, M, 16, 2040)
    work = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    n = ints(lengths)

    def call(i, s):
        tsfm.tsfm_tree_attention(s, pages, q[i], q[i].stride(1), out[i], out[i].stride(1), n, None, mask, depth, True, 3, M, 16, 0.09, 500, 4, 2040, None, work[i], size)

    for i in range(2):
        call(i, stream())
    torch.cuda.synchronize()
    want = [x.clone() for x in out]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for x in out:
            x.zero_()
        torch.cuda.synchronize()
        for i in range(2):
            call(i, streams[i].cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


# ------------------------------------------------------------------------------------------ what ordinary inputs do not reach
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,Hq,M", [(64, 4, 5), (64, 8, 40), (128, 16, 40), (128, 8, 70)])
@pytest.mark.parametrize("kind", ["spread", "low", "high", "rising"])
def test_scores_far_from_ordinary(dtype, D, Hq, M, kind):
    """Maxima that move by hundreds from tile to tile, scores that all lie far below or above 0."""
    lengths = [0, 70, 300]
    pool = Pool(3, 2, D, 16, [n + M for n in lengths], dtype, seed=8)
    trees = [tr.tree("random", M, b) for b in range(3)]
    if kind in ("low", "high"):
        pool.k[..., 0] = -40.0 if kind == "low" else 40.0
    if kind == "rising":                                       # the later a slot the larger its scores
        for b, n in enumerate(lengths):
            for s in range(n + M):
                pool.k[pool.table[b, s // 16].long(), :, s % 16, 0] = s / 4.0
    q = wide((3, M), Hq * D, dtype, 0, 2, 30.0 if kind == "spread" else 1.0)
    if kind != "spread":
        q.view(3, M, Hq, D)[..., 0] = 60.0
    tsfm = lib()
    for masks in ([tr.ancestors(t) for t in trees], None):
        out, lse = torch.zeros_like(q), torch.zeros(3, M, Hq, device="cuda")
        pages, ws = pool.describe(tsfm), torch.empty(1 << 25, dtype=torch.uint8, device="cuda")
        args = (stream(), pages, q, q.stride(1), out, out.stride(1), ints(lengths), None)
        if masks:
            tsfm.tsfm_tree_attention(*args, torch.stack([tr.words(s) for s, _ in masks]).cuda(), ints(np.stack([d for _, d in masks])), False, 3, M, Hq, 0.125, 0, 0,
                                     300 + M, lse, ws, ws.numel())
        else:
            tsfm.tsfm_window_attention(*args, 3, M, Hq, 0.125, 90, 4, 300 + M, lse, ws, ws.numel())
        for b, n in enumerate(lengths):
            k, v = pool.rows(pool.k, b, n + M), pool.rows(pool.v, b, n + M)
            for m in range(0, M, 3):
                seen = tr.visible(n, M, m, 0, 0, *masks[b]) if masks else tr.visible(n, M, m, 90, 4)
                o, z, absv, peak, count = tr.attention(q[b, m].cpu().double().view(Hq, D), k, v, 0.125, seen)
                rel = ref.attention_tolerance(dtype, D, count, peak)[:, None]
                assert ((out[b, m].cpu().double().view(Hq, D) - o).abs() <= U[dtype] * o.abs() + rel * absv + 1e-30).all(), (b, m)
                assert ((lse[b, m].cpu().double() - z).abs() <= rel[:, 0] + 4 * U[F32] * (z.abs() + peak + 1)).all(), (b, m)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M", [5, 40])
@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0])
def test_any_scale(dtype, M, scale):
    pool = Pool(2, 2, 64, 16, [100 + M, M], dtype, seed=9)
    trees = [tr.tree("random", M, b) for b in range(2)]
    for b, n in enumerate([100, 0]):
        stale(pool, b, n + M)
    check(pool, dtype, 8, 2, 64, [100, 0], [M, M], M, trees, scale=scale, window=30, sinks=2)
    check(pool, dtype, 8, 2, 64, [100, 0], [M, M], M, None, scale=scale)


@pytest.mark.parametrize("M", [5, 60])
def test_depths_are_cut(M):
    rng = np.random.default_rng(1)
    lengths = [100, 30]
    masks, cut = [], []
    for b in range(2):
        sees, _ = tr.ancestors(tr.tree("random", M, b))
        depth = rng.choice([-5, -2 ** 31, 2 ** 31 - 1, M, 1], M)
        masks.append((sees, depth))
        cut.append((sees, np.clip(depth, 0, M - 1)))
    pool = Pool(2, 2, 64, 16, [n + M for n in lengths], BF16, seed=1)
    a = check(pool, BF16, 8, 2, 64, lengths, [M, M], M, masks=cut, window=20, sinks=1)
    tsfm = lib()
    q = wide((2, M), 8 * 64, BF16, 0, 1, 2.0)                  # as check() makes them
    out, ws = torch.zeros_like(q), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    tsfm.tsfm_tree_attention(stream(), pool.describe(tsfm), q, q.stride(1), out, out.stride(1), ints(lengths), None, torch.stack([tr.words(s) for s, _ in masks]).cuda(),
                             ints(np.stack([d for _, d in masks])), False, 2, M, 8, 0.125, 20, 1, max(lengths) + M, None, ws, ws.numel())
    assert torch.equal(out, a[0][..., :8 * 64])


@pytest.mark.parametrize("M,Hq,D,page", [(1, 4, 64, 16), (40, 8, 64, 16), (40, 8, 128, 64), (70, 16, 128, 8)])
def test_a_wait_that_runs_out_ends_the_call(M, Hq, D, page):
    """Waits for more bytes than are copied (nothing faults, the copies themselves arrive): the status says so, NaN where it matters, and the next call is
    whole again."""
    tsfm = lib()
    lengths = [500, 200]
    pool = Pool(2, 2, D, page, [n + M for n in lengths], BF16, seed=3)
    q = wide((2, M), Hq * D, BF16, 0, 1)
    pages = pool.describe(tsfm)
    size = tsfm.tsfm_tree_attention_workspace(pages, 2, M, Hq, 500 + M)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def run():
        out = torch.zeros_like(q)
        tsfm.tsfm_window_attention(stream(), pages, q, q.stride(1), out, out.stride(1), ints(lengths), None, 2, M, Hq, 0.125, 0, 0, 500 + M, None, ws, size)
        torch.cuda.synchronize()
        return out

    good = run()
    try:
        tsfm.tsfm_debug_tile_wait(2000, 0)
        bad = run()
    finally:
        tsfm.tsfm_debug_tile_wait()
    assert int(pool.status) == tsfm.TSFM_PAGES_TIMEOUT and torch.isnan(bad.float()).all()
    pool.status.zero_()
    assert torch.equal(run(), good) and int(pool.status) == 0


def test_a_captured_call_follows_new_lengths_and_trees():
    """What a graph replays reads lengths, counts, masks and tables as they are then."""
    tsfm = lib()
    M, Hq, D = 40, 8, 64
    pool = Pool(2, 2, D, 16, [400, 400], BF16, seed=3)
    q = wide((2, M), Hq * D, BF16, 0, 1)
    pages = pool.describe(tsfm)
    size = tsfm.tsfm_tree_attention_workspace(pages, 2, M, Hq, 400)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    length, new = ints([10, 300]), ints([M, M])
    parent = ints([tr.tree("random", M, b) for b in range(2)])
    mask, depth = torch.zeros(2, M, 1, dtype=torch.int64, device="cuda"), torch.zeros(2, M, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)

    def call(to, work):
        tsfm.tsfm_tree_init(stream(), parent, new, 2, M, 0, mask, depth)
        tsfm.tsfm_tree_attention(stream(), pages, q, q.stride(1), to, to.stride(1), length, new, mask, depth, False, 2, M, Hq, 0.125, 50, 2, 400, None, work, size)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call(out, ws)
    for lengths, counts, seed in (([10, 300], [M, M], 0), ([0, 350], [7, 0], 5), ([359, 1], [M, 33], 9)):
        length.copy_(ints(lengths))
        new.copy_(ints(counts))
        parent.copy_(ints([tr.tree("random", M, seed + b) for b in range(2)]))
        out.fill_(-3)
        graph.replay()
        want = torch.full_like(out, -3)
        call(want, torch.empty_like(ws))
        torch.cuda.synchronize()
        assert torch.equal(out, want)
