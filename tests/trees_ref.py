"""Trees of drafted tokens, windows with sinks and log probabilities in 64 bits, from the definitions (include/tsfm.h)."""
import math

import numpy as np
import torch

from tests import serving_ref as ref


def tree(kind, M, seed):
    """Parents of M nodes, node 0 the root.  "loose" has further roots among them."""
    rng = np.random.default_rng(seed)
    if kind == "chain":
        return [m - 1 for m in range(M)]
    if kind == "star":
        return [-1] + [0] * (M - 1)
    if kind == "binary":
        return [(m - 1) // 2 if m else -1 for m in range(M)]
    return [-1] + [int(rng.integers(-1 if kind == "loose" else 0, m)) for m in range(1, M)]


def ancestors(parent, window=0):
    """(sees [M, M], depth [M]) of a tree."""
    M = len(parent)
    sees, depth = np.zeros((M, M), bool), np.zeros(M, np.int64)
    for m in range(M):
        chain, i = [], m
        while i >= 0:
            chain.append(i)
            i = parent[i] if -1 <= parent[i] < i else -1
        depth[m] = len(chain) - 1
        sees[m, chain[:window] if window else chain] = True
    return sees, depth


def words(sees):
    """[M, ceil(M / 64)] int64 of a matrix of truth values."""
    M = sees.shape[1]
    bits = np.zeros((sees.shape[0], (M + 63) // 64), np.uint64)
    for j in range(M):
        bits[:, j // 64] |= sees[:, j].astype(np.uint64) << np.uint64(j % 64)
    return torch.from_numpy(bits.view(np.int64).copy())


def visible(length, new, m, window, sinks, sees=None, depth=None):
    """[length + new] of truth values: what token m sees; sees None: a chain."""
    s = np.arange(length + new)
    if sees is None:
        return (s <= length + m) & ((s > length + m - window) if window else True) | (s < min(sinks if window else 0, length + m + 1))
    old = (s[:length] > length + depth[m] - window) | (s[:length] < sinks) if window else np.ones(length, bool)
    return np.concatenate([old, sees[m, :new]])


def attention(q, k, v, scale, seen):
    """One token: q [Hq, D], k and v [n, Hkv, D] fp64, seen [n].  (out [Hq, D], lse [Hq], the sum of p |v|, the largest sum of |q k| scale, slots)."""
    idx = torch.from_numpy(np.flatnonzero(seen))
    o, z, _, absv, peak = ref.attention(q, k[idx], v[idx], scale, 0, len(idx))
    return o, z, absv, peak, len(idx)


def logprobs(x, scale, tokens, n):
    """One row: (logprob of tokens, lse, entropy, ids, their logprob) of logits x (1-D, any float type)."""
    raw = x.double()
    y = raw * scale
    gone = bool((y == -math.inf).all())
    bad = bool(torch.isnan(y).any()) or bool((y == math.inf).any())
    # relative to the largest: logits of the type's lowest value leave nothing of log V beside them, in 64 bits either
    top = 0.0 if gone else float(y.max())
    d = y - top
    log_sum = -math.inf if gone else math.nan if bad else math.log(float(d.exp().sum()))
    z = top + log_sum
    log_p = d - log_sum
    entropy = 0.0 if gone else math.nan if bad else -float(torch.where(log_p > -math.inf, log_p.exp() * log_p, torch.zeros_like(d)).sum())
    minus = lambda t: -math.inf if gone else float(log_p[t])
    order = sorted(range(len(y)), key=lambda t: (math.isnan(raw[t]), -float(raw[t]) if not math.isnan(raw[t]) else 0.0, t)) if len(y) < 2000 else \
        np.lexsort((np.arange(len(y)), -raw.numpy())).tolist()
    ids = order[:n] + [-1] * max(0, n - len(y))
    return [minus(t) if 0 <= t < len(y) else -math.inf for t in tokens], z, entropy, ids, [minus(t) if t >= 0 else -math.inf for t in ids]


def rest(p, q, used, gone):
    """What is left of a node's row: weights of the draw."""
    if q is not None:
        return np.maximum(p - used * q, 0.0)
    r = p.copy()
    r[list(gone)] = 0.0
    return r


def verify(tokens, parent, p, q, u, nodes):
    """One series: tokens [M], parent [M], p, q [M, V] (weights), u [M + 1].  (committed tokens, path)."""
    if nodes == 0:
        return [], []
    V = p.shape[1]
    cut = lambda x: 0.0 if math.isnan(x) else min(max(float(x), 0.0), 1.0 - 2.0 ** -24)
    here, path = 0, [0]
    while True:
        used, mass, gone, reached = 0.0, 1.0, set(), None
        for j in range(here + 1, nodes):
            if parent[j] != here:
                continue
            x = int(tokens[j])
            inside = 0 <= x < V
            r = rest(p[here], None if q is None else q[here], used, gone)
            qx = 1.0 if q is None else float(q[here, x]) if inside else 1.0
            if inside and cut(u[j]) * qx * mass < r[x]:
                reached = j
                break
            if q is None:
                if inside:
                    mass -= float(r[x])
                    gone.add(x)
            else:
                used += mass
                mass = math.fsum(rest(p[here], q[here], used, gone))
        if reached is None:
            break
        path.append(reached)
        here = reached
    r = rest(p[here], None if q is None else q[here], used, gone)
    if not r.sum() > 0:
        r = p[here]
    return [int(tokens[j]) for j in path[1:]] + [ref.draw(r, float(u[-1]))], path
