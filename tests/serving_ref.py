"""Serving over a cache of pages in 64 bits, slot by slot from the definitions (include/tsfm.h), and inputs for its tests."""
import math

import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}          # half a step of a rounding, relative


class Pool:
    """A pool of pages with a table for B series of `slots` slots; pages shuffled, -1 behind a series' last page.
    order "heads": [page, head, slot, D]; "slots": [page, slot, head, D]."""

    def __init__(self, B, Hkv, D, page, slots, dtype, order="heads", seed=0, spare=0, fill=None, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        counts = [-(-int(s) // page) for s in slots]
        total = max(1, sum(counts) + spare)
        perm = torch.randperm(total, generator=g).tolist()
        self.page, self.B = page, B
        self.table = torch.full((B, max(1, max(counts))), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(counts):
            self.table[b, :n] = torch.tensor(perm[at:at + n], dtype=torch.int32)
            at += n
        self.spare_ids = perm[at:]
        shape = (total, Hkv, page, D) if order == "heads" else (total, page, Hkv, D)
        make = lambda: (torch.full(shape, fill) if fill is not None else torch.randn(shape, generator=g)).to(dtype).to(device)
        self.k, self.v = make(), make()
        if order != "heads":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.table = self.table.to(device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def describe(self, tsfm, table=None):
        return tsfm.kv_pages(self.k, self.v, self.table if table is None else table, self.status)

    def rows(self, x, b, n, table=None):
        """[n, Hkv, D] in fp64: slots 0..n-1 of series b of pool x (k or v)."""
        t = (self.table if table is None else table)[b].cpu().long()
        s = torch.arange(n)
        return x.cpu()[t[s // self.page], :, s % self.page].double()

    def put(self, x, b, slot, value):
        x[self.table[b, slot // self.page].long(), :, slot % self.page] = value


def frequencies(rot, base, scaling, factor=1.0, original=0.0, lo=0.0, hi=0.0):
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2.0))
    f = base ** (-2.0 * i / max(rot, 1))
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        g = np.clip((original * f / (2 * math.pi) - lo) / (hi - lo), 0, 1)
        f = f * (g + (1 - g) / factor)
    return f


def turn(x, pos, f, layout, mscale=1.0):
    """x [heads, D] fp64 at position pos."""
    n = len(f)
    i = np.arange(n)
    a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
    c, s = torch.from_numpy(np.cos(pos * f)), torch.from_numpy(np.sin(pos * f))
    y = x.clone()
    y[:, a], y[:, b] = mscale * (x[:, a] * c - x[:, b] * s), mscale * (x[:, a] * s + x[:, b] * c)
    return y


def attention(q, k, v, scale, start, end):
    """One token: q [Hq, D], k and v [n, Hkv, D] fp64, slots start <= s < end.  (out [Hq, D], lse [Hq], p [Hq, n], the sum of
    p |v| [Hq, D], the largest sum of |q k| scale [Hq])."""
    Hq, D = q.shape
    n, Hkv, _ = k.shape
    G = Hq // Hkv
    p, absv, peak = torch.zeros(Hq, n, dtype=torch.float64), torch.zeros(Hq, D, dtype=torch.float64), torch.zeros(Hq, dtype=torch.float64)
    if end <= start:
        return torch.zeros(Hq, D, dtype=torch.float64), torch.full((Hq,), -math.inf, dtype=torch.float64), p, absv, peak
    kk, vv = k[start:end].repeat_interleave(G, 1), v[start:end].repeat_interleave(G, 1)      # [n, Hq, D]
    score = torch.einsum("hd,nhd->hn", q, kk) * scale
    peak = torch.einsum("hd,nhd->hn", q.abs(), kk.abs()).amax(1) * abs(scale)
    lse = torch.logsumexp(score, 1)
    w = torch.exp(score - lse[:, None])
    p[:, start:end] = w
    return torch.einsum("hn,nhd->hd", w, vv), lse, p, torch.einsum("hn,nhd->hd", w, vv.abs()), peak


def attention_tolerance(dtype, D, n, peak):
    """Relative error of a probability in 32 bits: a dot of D products (D + 1 roundings of partial sums that |q||k| bounds, and
    the scale's), the exponential (2 steps and its argument's rounding, |score - max| <= 2 peak), a sum of n; once for p, once
    for the sum.  bf16 kernels may round p to bf16 for the product with the values."""
    score = (D + 3) * U[torch.float32] * peak
    return 2 * (score + (4 + 4 * peak) * U[torch.float32]) + (n + 8) * U[torch.float32] + (U[torch.bfloat16] if dtype == torch.bfloat16 else 0)


def evict(w, n, budget, sinks, recent):
    """Slots that are kept, ascending."""
    if n <= budget:
        return list(range(n))
    middle = list(range(sinks, n - recent))
    rank = lambda s: -math.inf if math.isnan(w[s]) else float(w[s])
    # NaN below -inf
    best = sorted(middle, key=lambda s: (math.isnan(w[s]), -rank(s), s))[:budget - sinks - recent]
    return sorted(list(range(sinks)) + best + list(range(n - recent, n)))


def weight(x):
    x = np.asarray(x, np.float64)
    return np.where(np.isfinite(x) & (x > 0), x, 0.0)


def draw(r, u):
    """Smallest t with the running sum above u times the total; exact rational sums (math.fsum) decide."""
    r = np.asarray(r, np.float64)
    c = np.cumsum(r)
    if not c[-1] > 0:
        return -1
    u = 0.0 if math.isnan(u) else min(max(float(u), 0.0), 1.0 - 2.0 ** -24)
    t = int(np.searchsorted(c, u * c[-1], side="right"))
    return min(t, int(np.nonzero(r)[0][-1]))


def verify(tokens, p, q, u, nd):
    """One series: tokens [K], p [K+1, V], q [K, V] or None, u [K+1].  (committed tokens, n)."""
    V = p.shape[1]
    n = nd
    for i in range(nd):
        x = int(tokens[i])
        ok = False
        if 0 <= x < V:
            ui = 0.0 if math.isnan(u[i]) else min(max(float(u[i]), 0.0), 1.0 - 2.0 ** -24)
            qx = 1.0 if q is None else float(weight(q[i, x]))
            ok = ui * qx < float(weight(p[i, x]))
        if not ok:
            n = i
            break
    w = weight(p[n])
    if n < nd:
        if q is None:
            d = np.zeros(V)
            if 0 <= int(tokens[n]) < V:
                d[int(tokens[n])] = 1.0
        else:
            d = weight(q[n])
        r = np.maximum(w - d, 0.0)
        if not r.sum() > 0:
            r = w
    else:
        r = w
    return [int(t) for t in tokens[:n]] + [draw(r, float(u[len(u) - 1]))], n
