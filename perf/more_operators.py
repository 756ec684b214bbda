"""Operators of a served model that drafts trees of tokens, one call each: attention of a tree, or of a chain within a sliding window,
over a cache of pages, with first slots that stay visible; log probabilities, entropy and best tokens of logits; verification
of a drafted tree; commit of its accepted path in the cache.

Caches are pools of pages [page, kv head, slot, d_head] (the commit's: [layer, page, kv head, slot, d_head]); a series' slot s lies
in page table[b, s // page_size].  Lengths, accepted tokens and the like are spread over a batch by rank, so that work(case)
follows from the case alone; the seed decides which series has which.  A tree is given by parents, parent[m] < m, node 0 the
last committed token; bit j of a node's mask says that it sees node j, and bits go in words of 64.

`own` False computes the operators from elementary torch operations in 32 bits (cumulated probabilities in 64).
"""
import math

import numpy as np
import torch

own = False

F32, BF16 = "f32", "bf16"
TORCH = {F32: torch.float32, BF16: torch.bfloat16}
BYTES = {F32: 4, BF16: 2}


# ------------------------------------------------------------------------------------------ cases
def _attend(op, name, dtype, B, M, Hq, Hkv, D, page, longest, skew, window=0, sinks=0, chain=0.0, shared=False):
    """longest: slots of the longest series with the new tokens, skew: how lengths fall off; chain: share of a tree's nodes
    that hang on the node before them; shared: one tree for all series."""
    c = dict(op=op, dtype=dtype, B=B, M=M, Hq=Hq, Hkv=Hkv, D=D, page=page, longest=longest, skew=skew, window=window, sinks=sinks)
    if op == "tree":
        c.update(chain=chain, shared=shared)
    return dict(c, name=name) if name else c


def _logprobs(name, dtype, rows, V, pad, tokens, top, temperature, masked):
    """pad: elements between rows; masked: a share of each row is -inf."""
    c = dict(op="logprobs", dtype=dtype, rows=rows, V=V, pad=pad, tokens=tokens, top=top, temperature=temperature, masked=masked)
    return dict(c, name=name) if name else c


def _verify(name, B, M, V, sampled, chain):
    c = dict(op="verify", B=B, M=M, V=V, sampled=sampled, chain=chain)
    return dict(c, name=name) if name else c


def _commit(name, dtype, layers, B, M, Hkv, D, page, ctx, longest):
    """ctx: longest length before the tree; longest: tokens of the longest path."""
    c = dict(op="commit", dtype=dtype, layers=layers, B=B, M=M, Hkv=Hkv, D=D, page=page, ctx=ctx, longest=longest)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a few candidates behind one short series, the smallest models (fp32): latency
        _attend("tree", "tree-one", F32, 1, 7, 4, 4, 32, 16, 38, 0.0, chain=0.3),
        # a static tree for all series, the 500 M model's heads and capacity
        _attend("tree", "tree-verification", BF16, 64, 26, 20, 20, 64, 16, 346, 0.25, chain=0.4, shared=True),
        # a tree for each series of a serving batch, grouped heads, long contexts
        _attend("tree", "tree-large", BF16, 32, 61, 32, 8, 128, 32, 8192, 1.0, chain=0.4),
        # one token of one endless stream
        _attend("window", "window-one", BF16, 1, 1, 32, 8, 128, 64, 70001, 0.0, window=4096, sinks=4),
        # a serving batch of them, one token each, some shorter than the window
        _attend("window", "window-batch", BF16, 256, 1, 32, 8, 128, 32, 8192, 2.0, window=1024, sinks=4),
        # prompts, all of their tokens at once
        _attend("window", "window-prompts", BF16, 4, 4096, 32, 8, 128, 64, 8192, 0.5, window=1024, sinks=4),
        # what a server returns for the token of one series
        _logprobs("logprobs-one", F32, 1, 32003, 0, 1, 5, 1.0, False),
        # scoring of many tokens, a large vocabulary, rows that begin anywhere
        _logprobs("logprobs-batch", BF16, 2048, 100003, 0, 1, 10, 0.8, False),
        # a small tree of one series
        _verify("verify-tree-one", 1, 8, 32003, True, 0.3),
        # a batch of trees, a large vocabulary
        _verify("verify-tree-batch", 64, 33, 100003, True, 0.4),
        # the path of one series in every layer of a small model (fp32)
        _commit("commit-one", F32, 4, 1, 16, 4, 64, 16, 120, 5),
        # a serving batch, all layers
        _commit("commit-batch", BF16, 24, 64, 61, 8, 128, 32, 200, 9),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


LARGEST = {"tree": (0.6e9, 160e9), "window": (0.7e9, 300e9), "logprobs": (0.42e9, 1e12), "verify": (0.2e9, 1e12), "commit": (0.2e9, 1e12)}
POOL = 256 * 8192 * 8 * 128                                # elements of a cache
DENSE = 1 << 32                                            # scores in a plain form


def _drawn(rng):
    op = rng.choice(["tree", "tree", "window", "window", "logprobs", "verify", "commit"])
    if op == "logprobs":
        return _logprobs(None, rng.choice([F32, BF16]), _log_int(rng, 1, 2048), _log_int(rng, 100, 131072), rng.choice([0, 0, 1, 8, 13]),
                         rng.choice([0, 1, 1, 4, 17]), rng.choice([0, 1, 5, 10, 20, 32]), rng.choice([1.0, 0.7, 1.5]), rng.random() < 0.3)
    if op == "verify":
        return _verify(None, _log_int(rng, 1, 64), _log_int(rng, 1, 64), _log_int(rng, 100, 131072), rng.random() < 0.7, rng.choice([0.0, 0.4, 0.8]))
    dtype, D, page = rng.choice([F32, BF16, BF16, BF16]), rng.choice([32, 64, 128]), rng.choice([8, 16, 32, 64, 128])
    Hkv = rng.choice([1, 2, 4, 5, 8])
    if op == "commit":
        M = _log_int(rng, 4, 128)
        return _commit(None, dtype, _log_int(rng, 1, 32), _log_int(rng, 1, 64), M, Hkv, D, page, _log_int(rng, 1, 400), rng.randint(2, min(M // 2, 16)))
    Hq = Hkv * rng.choice([1, 2, 3, 4, 8])
    longest, skew, sinks = _log_int(rng, 1, 65536), rng.choice([0.0, 0.25, 1.0, 2.0]), rng.choice([0, 1, 4, 70])
    if op == "tree":
        return _attend(op, None, dtype, _log_int(rng, 1, 64), _log_int(rng, 1, 128), Hq, Hkv, D, page, longest, skew,
                       window=rng.choice([0, 0, _log_int(rng, 1, longest)]), sinks=sinks, chain=rng.choice([0.0, 0.4, 0.8]), shared=rng.random() < 0.5)
    M = rng.choice([1, 1, 2, 5, 9, _log_int(rng, 16, 4096)])
    return _attend(op, None, dtype, _log_int(rng, 1, 256 if M < 16 else 8), M, Hq, Hkv, D, page, longest, skew,
                   window=_log_int(rng, 1, 4096), sinks=sinks)


def _pool(c):
    return sum(_lengths(c)) * c["Hkv"] * c["D"]


def draw(rng):
    while True:
        c = _drawn(rng)
        w = work(c)
        most = LARGEST[c["op"]]
        if w["bytes"] > most[0] or w["flops"] > most[1] * (0.02 if c.get("dtype") == F32 and c["op"] in ("tree", "window") else 1.0):
            continue
        if c["op"] in ("tree", "window") and (_pool(c) > POOL or c["Hq"] * min(c["M"], BLOCK) * (_span(c) + BLOCK) * c["B"] > DENSE):
            continue
        if c["op"] == "verify" and c["B"] * c["M"] * c["V"] > 64 * 33 * 100003:
            continue
        if c["op"] == "commit" and c["layers"] * c["B"] * (c["ctx"] + c["M"] + c["page"]) * c["Hkv"] * c["D"] > 1 << 29:
            continue
        return c


def _lengths(c):
    """Slots of each series with the new tokens, in ascending order of rank."""
    return [int(round(c["longest"] * ((i + 1) / c["B"]) ** c["skew"])) for i in range(c["B"])]


def _new(c):
    """New tokens of each series by rank: every fourth one of a batch has fewer, some none."""
    return [min(n, c["M"] if i % 4 != 3 else c["M"] * (i % 7) // 7) for i, n in enumerate(_lengths(c))]


def _span(c):
    """Slots before the new tokens that the longest series' tokens see."""
    return min(c["longest"], c["sinks"] + c["window"]) if c["window"] else c["longest"]


def _paths(c):
    """Committed tokens of each series by rank, the root among them."""
    return [1 + (c["longest"] - 1) * ((5 * i + 3) % 8) // 7 for i in range(c["B"])]


def work(c):
    if c["op"] == "logprobs":
        per = BYTES[c["dtype"]] * c["V"] + c["tokens"] * 8 + c["top"] * 8 + 8
        return {"bytes": float(c["rows"] * per), "flops": c["rows"] * c["V"] * 6.0}
    if c["op"] == "verify":
        # a row of the target's probabilities a series and with sampled drafts one of the draft's; where a child is rejected, its entries
        rows = 2.0 if c["sampled"] else 1.0
        return {"bytes": c["B"] * (c["V"] * 4.0 * rows + c["M"] * 24.0), "flops": c["B"] * c["V"] * rows}
    e = BYTES[c["dtype"]]
    if c["op"] == "commit":
        moved = sum(p - 1 for p in _paths(c))
        return {"bytes": c["layers"] * moved * c["Hkv"] * c["D"] * 4.0 * e + c["B"] * (c["M"] + 1) * 4.0, "flops": 0.0}
    total, new = _lengths(c), _new(c)
    read = pairs = 0
    for n, k in zip(total, new):
        before = n - k
        if c["op"] == "tree":
            prefix = min(before, c["sinks"] + c["window"]) if c["window"] else before
            read += (prefix + k) if k else 0
            pairs += k * (prefix + 1)
        else:
            first = max(0, min(before, before + 1 - c["window"]))                       # first slot in the first token's window
            read += (n - first + min(first, c["sinks"])) if k else 0
            # token m sees its window, the sinks before it
            ends = np.arange(before + 1, n + 1, dtype=np.int64)
            starts = np.maximum(0, ends - c["window"])
            pairs += int((ends - starts + np.minimum(starts, c["sinks"])).sum())
    b = read * c["Hkv"] * c["D"] * 2.0 * e + sum(new) * c["Hq"] * (2.0 * c["D"] * e + 4) + c["B"] * 8
    return {"bytes": b, "flops": pairs * c["Hq"] * 4.0 * c["D"]}


# ------------------------------------------------------------------------------------------ inputs
def _int(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _pages(page, slots, order):
    """A table [B, most pages] for series of `slots` slots each, the pages in a shuffled order, and the pool's size."""
    counts = [-(-s // page) for s in slots]
    most, total = max(1, max(counts)), max(1, sum(counts))
    perm = order.permutation(total).astype(np.int32)
    table = np.full((len(slots), most), -1, np.int32)
    at = 0
    for row, k in zip(table, counts):
        row[:k] = perm[at:at + k]
        at += k
    return torch.from_numpy(table).cuda(), total


def _tree(order, M, chain):
    """Parents of M nodes, node 0 the root."""
    parent = np.full(M, -1, np.int32)
    for m in range(1, M):
        parent[m] = m - 1 if order.random_sample() < chain else order.randint(0, m)
    return parent


def _ancestors(parent):
    """[M, M] of truth values (a node sees itself and its ancestors), depths."""
    M = len(parent)
    sees, depth = np.eye(M, dtype=bool), np.zeros(M, np.int32)
    for m in range(M):
        if parent[m] >= 0:
            sees[m] |= sees[parent[m]]
            depth[m] = depth[parent[m]] + 1
    return sees, depth


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    order = np.random.RandomState(seed % (1 << 32))
    s = {"case": c}
    if c["op"] == "logprobs":
        return _prepare_logprobs(s, c, g)
    if c["op"] == "verify":
        return _prepare_verify(s, c, g, order)
    t, B, Hkv, D, page = TORCH[c["dtype"]], c["B"], c["Hkv"], c["D"], c["page"]
    which = order.permutation(B)

    def normal(*shape):
        return torch.empty(shape, dtype=t, device="cuda").normal_(generator=g)

    if c["op"] == "commit":
        ctx = [c["ctx"] * (i + 1) // B for i in which]
        s["table"], n = _pages(page, [x + c["M"] for x in ctx], order)
        s["k"], s["v"] = (normal(c["layers"], n, Hkv, page, D) for _ in "kv")
        # nodes are numbered level by level: the first of a path lies behind as many as the path is long, where there are as many
        path = np.full((B, c["M"]), -1, np.int32)
        for row, i in zip(path, which):
            p = _paths(c)[i]
            row[0] = 0
            row[1:p] = np.sort(order.choice(np.arange(p, c["M"]), p - 1, replace=False))
        s["path"], s["len"] = _int(path), _int(ctx)
        return s
    total, new = [_lengths(c)[i] for i in which], [_new(c)[i] for i in which]
    M, Hq = c["M"], c["Hq"]
    s["table"], n = _pages(page, total, order)
    s["n_new"], s["len"] = _int(new), _int([x - y for x, y in zip(total, new)])
    s["k"], s["v"] = (normal(n, Hkv, page, D) for _ in "kv")
    s["q"] = normal(B, M, Hq * D) * 2                       # scores of standard deviation 2: neither flat nor one slot
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(B, M, Hq, device="cuda")
    if c["op"] == "tree":
        trees = [_tree(order, M, c["chain"]) for _ in range(1 if c["shared"] else B)]
        sees, depth = zip(*(_ancestors(p) for p in trees))
        s["parent"], s["depth"], s["sees"] = _int(trees), _int(depth), torch.from_numpy(np.stack(sees)).cuda()
    return s


def _prepare_logprobs(s, c, g):
    rows, V = c["rows"], c["V"]
    wide = torch.empty(rows, V + c["pad"], dtype=TORCH[c["dtype"]], device="cuda").normal_(generator=g)
    x = wide[:, :V]
    x.mul_(2.5)
    # a few tokens stand out
    at = torch.randint(0, V, (rows, 8), generator=g, device="cuda")
    x.scatter_(1, at, (torch.rand(rows, 8, generator=g, device="cuda") * 12 + 6).to(x.dtype))
    if c["masked"]:                                         # a grammar forbids most tokens of some rows and a few of the others
        share = torch.where(torch.arange(rows, device="cuda") % 3 == 0, 0.95, 0.05)[:, None]
        for r in range(0, rows, 256):
            x[r:r + 256].masked_fill_(torch.rand(x[r:r + 256].shape, generator=g, device="cuda") < share[r:r + 256], -math.inf)
    s["logits"] = x
    s["tokens"] = torch.randint(0, V, (rows, c["tokens"]), generator=g, device="cuda", dtype=torch.int32)
    s["logprob"], s["lse"], s["entropy"] = torch.zeros(rows, c["tokens"], device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    s["ids"], s["best"] = torch.zeros(rows, c["top"], dtype=torch.int32, device="cuda"), torch.zeros(rows, c["top"], device="cuda")
    return s


def _prepare_verify(s, c, g, order):
    B, M, V = c["B"], c["M"], c["V"]

    def probabilities(x):                                   # as samplers cut them: tokens that are all but impossible are
        p = torch.softmax(x, -1)
        p = torch.where(p < 0.02 / V, torch.zeros_like(p), p)
        return p / p.sum(-1, keepdim=True)

    trees = np.stack([_tree(order, M, c["chain"]) for _ in range(B)])
    new = np.array([M if i % 4 != 3 else M * (i % 7) // 7 for i in range(B)])[order.permutation(B)]
    s["parent"], s["n_new"] = _int(trees), _int(new)
    # a draft that tracks its target, and its children drawn from it, or its best tokens
    x = torch.randn(B, M, V, generator=g, device="cuda") * 2.5
    q = probabilities(x)
    x += 0.5 * torch.randn(x.shape, generator=g, device="cuda")
    s["p"] = probabilities(x)
    del x
    up = s["parent"].long().clamp(min=0)
    rows = q.view(B * M, V)
    if c["sampled"]:
        drawn = torch.multinomial(rows, M, replacement=True, generator=g).view(B, M, M)      # [b, node, its m-th draw]
    else:
        best = rows.topk(min(M, V)).indices
        drawn = torch.nn.functional.pad(best, (0, M - best.shape[1])).view(B, M, M)
        nth = np.zeros((B, M), np.int64)                    # number of a node among its siblings
        for b in range(B):
            count = np.zeros(M, np.int64)
            for m in range(1, M):
                nth[b, m] = count[trees[b, m]]
                count[trees[b, m]] += 1
    at = torch.arange(M, device="cuda").expand(B, M) if c["sampled"] else torch.from_numpy(nth).cuda()
    s["tokens"] = drawn[torch.arange(B, device="cuda")[:, None], up, at].int()
    s["q"] = q if c["sampled"] else None
    s["u"] = torch.rand(B, M + 1, generator=g, device="cuda")
    s["len"] = torch.randint(1, 5000, (B,), generator=g, device="cuda", dtype=torch.int32)
    s["out"], s["path"] = (torch.zeros(B, M, dtype=torch.int32, device="cuda") for _ in range(2))
    s["n_accept"], s["len_out"] = torch.zeros_like(s["len"]), torch.zeros_like(s["len"])
    return s


# ------------------------------------------------------------------------------------------ plain forms
BLOCK = 512                                                # tokens of a prompt that are looked at together


def _run_attend(s):
    """Tokens in blocks; of each block only the slots that a token of it may see."""
    c = s["case"]
    B, M, Hq, Hkv, D, page = (c[k] for k in ("B", "M", "Hq", "Hkv", "D", "page"))
    G = Hq // Hkv
    out, lse = s["out"].clone(), s["lse"].clone()
    length, new = s["len"].long(), s["n_new"].long()
    tree = c["op"] == "tree"
    for m0 in range(0, M, BLOCK):
        m = torch.arange(m0, min(M, m0 + BLOCK), device="cuda")
        # columns: the sinks, then the slots from the first one in a window on (all of them without one)
        first = (length + m0 + 1 - c["window"]).clamp(min=0) if c["window"] else torch.zeros_like(length)
        if tree:
            first = torch.minimum(first, length)
        sinks = c["sinks"] if c["window"] else 0
        wide = min(c["longest"], (c["window"] + len(m) - 1 if not tree else c["window"] + M) if c["window"] else c["longest"])
        columns = torch.cat([torch.arange(sinks, device="cuda").expand(B, sinks), first[:, None] + torch.arange(wide, device="cuda")], 1)
        once = torch.ones_like(columns, dtype=torch.bool)
        once[:, :sinks] = columns[:, :sinks] < first[:, None]           # (a sink within the window counts once)
        exists = once & (columns < (length + new)[:, None])
        position = length[:, None] + (s["depth"].long()[:, m] if tree else m)                      # [B or 1 -> B, m]
        low = position[..., None] - c["window"] if c["window"] else torch.full_like(position[..., None], -1)
        near = (columns[:, None] > low) | (columns[:, None] < c["sinks"])
        if tree:
            j = columns - length[:, None]
            bits = s["sees"].expand(B, M, M)[:, m].gather(2, j.clamp(0, M - 1)[:, None].expand(B, len(m), columns.shape[1]))
            seen = torch.where((j < 0)[:, None], near, bits)
        else:
            seen = near & (columns[:, None] <= position[..., None])
        live = (m < new[:, None])
        seen = seen & exists[:, None] & live[..., None]
        at = columns.clamp(0, s["table"].shape[1] * page - 1)
        ids = s["table"].long().gather(1, at // page).clamp(min=0)
        gone = ~seen.any(1)
        k, v = (x[ids, :, at % page].float().masked_fill_(gone[..., None, None], 0.0).transpose(1, 2) for x in (s["k"], s["v"]))
        q = s["q"][:, m].float().view(B, len(m), Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, len(m) * G, D)
        score = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(D))
        score.masked_fill_(~seen[:, None, :, None].expand(B, 1, len(m), G, columns.shape[1]).reshape(B, 1, len(m) * G, -1), -math.inf)
        top = score.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        p = (score - top).exp_()
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
        o = o.view(B, Hkv, len(m), G, D).permute(0, 2, 1, 3, 4).reshape(B, len(m), Hq * D)
        z = (top + total.log()).view(B, Hkv, len(m), G).permute(0, 2, 1, 3).reshape(B, len(m), Hq)
        out[:, m] = torch.where(live[..., None], o.to(out.dtype), out[:, m])
        lse[:, m] = torch.where(live[..., None], z, lse[:, m])
    return {"out": out, "lse": lse}


def _run_logprobs(s):
    c = s["case"]
    rows, V, top = c["rows"], c["V"], c["top"]
    out = {"logprob": torch.empty_like(s["logprob"]), "lse": torch.empty_like(s["lse"]), "entropy": torch.empty_like(s["entropy"]),
           "ids": torch.full_like(s["ids"], -1), "best": torch.full_like(s["best"], -math.inf)}
    for r in range(0, rows, 256):
        to = slice(r, r + 256)
        x = s["logits"][to].float() * (1.0 / c["temperature"])
        high = x.amax(1, keepdim=True)
        high = torch.where(high == -math.inf, torch.zeros_like(high), high)
        d = x - high
        e = d.exp()
        total = e.sum(1, keepdim=True)
        log_total = total.log()
        out["lse"][to] = (high + log_total)[:, 0]
        mean = torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1, keepdim=True)
        out["entropy"][to] = torch.where(total > 0, log_total - mean / total, torch.zeros_like(total))[:, 0]
        if c["tokens"]:
            out["logprob"][to] = d.gather(1, s["tokens"][to].long()) - log_total
        if top:
            n = min(top, V)
            best = torch.sort(s["logits"][to].float(), dim=1, descending=True, stable=True).indices[:, :n]
            out["ids"][to, :n] = best.int()
            out["best"][to, :n] = d.gather(1, best) - log_total
    return out


def _run_verify(s):
    """All trees a level and a child at a time: where series are done nothing changes any more."""
    c = s["case"]
    B, M, V = c["B"], c["M"], c["V"]
    b, node = torch.arange(B, device="cuda"), torch.arange(M, device="cuda")
    parent, tokens = s["parent"].long(), s["tokens"].long()
    here = torch.zeros(B, dtype=torch.long, device="cuda")              # the node that the walk has reached
    tried = torch.zeros_like(here)                                      # children of it up to here have been rejected
    level = torch.zeros_like(here)
    used = torch.zeros(B, dtype=torch.double, device="cuda")            # c_k
    mass = torch.ones(B, dtype=torch.double, device="cuda")             # Z_k
    out, path = torch.full_like(s["out"], -1), torch.full_like(s["path"], -1)
    idle = s["n_new"] <= 0
    path[:, 0] = torch.where(idle, path[:, 0], torch.zeros_like(path[:, 0]))
    removed = torch.zeros(B, V, dtype=torch.bool, device="cuda") if not c["sampled"] else None
    for _ in range(M):
        child = (parent == here[:, None]) & (node > tried[:, None]) & (node > here[:, None]) & (node < s["n_new"][:, None])
        some = child.any(1)
        x = torch.where(some, child.int().argmax(1), torch.zeros_like(here))
        token = tokens[b, x]
        u = s["u"][b, x].double()
        p = s["p"][b, here, token].double()
        if c["sampled"]:
            q = s["q"][b, here, token].double()
            ok = some & (u * q * mass < (p - used * q).clamp(min=0))
            no = some & ~ok
            used = torch.where(no, used + mass, used)
            rows = torch.where(no)[0]                       # (which rows: the next sum needs those alone)
            if len(rows):
                rest = (s["p"][rows, here[rows]].double() - used[rows, None] * s["q"][rows, here[rows]].double()).clamp_(min=0)
                mass[rows] = rest.sum(1)
        else:
            p = torch.where(removed[b, token], torch.zeros_like(p), p)
            ok = some & (u * mass < p)
            no = some & ~ok
            mass = torch.where(no, mass - p, mass)
            removed[b, token] |= no
            removed &= ~ok[:, None]
        level = torch.where(ok, level + 1, level)
        out[b, (level - 1).clamp(min=0)] = torch.where(ok, token.int(), out[b, (level - 1).clamp(min=0)])
        path[b, level] = torch.where(ok, x.int(), path[b, level])
        here, tried = torch.where(ok, x, here), torch.where(some, x, tried)
        used, mass = torch.where(ok, torch.zeros_like(used), used), torch.where(ok, torch.ones_like(mass), mass)
    p = s["p"][b, here].double()
    if c["sampled"]:
        rest = torch.where((used > 0)[:, None], (p - used[:, None] * s["q"][b, here].double()).clamp(min=0), p)
    else:
        rest = torch.where(removed, torch.zeros_like(p), p)
    rest = torch.where(rest.sum(1, keepdim=True) > 0, rest, p)
    cdf = rest.cumsum(1)
    t = (cdf <= s["u"][:, M:].double() * cdf[:, -1:]).sum(1)
    t = torch.minimum(t, V - 1 - (rest.flip(1) > 0).int().argmax(1))
    out[b, level] = torch.where(idle, out[b, level], t.int())
    return {"tokens": out, "path": path, "n_accept": level.int(), "len": torch.where(idle, s["len"], s["len"] + level.int() + 1)}


def _run_commit(s):
    c = s["case"]
    page = c["page"]
    b, i = (s["path"] > 0).nonzero(as_tuple=True)
    slot = s["len"].long()[b]
    source, target = slot + s["path"][b, i], slot + i
    ids = s["table"].long()
    source, target = (slice(None), ids[b, source // page], slice(None), source % page), (slice(None), ids[b, target // page], slice(None), target % page)
    for pool in (s["k"], s["v"]):
        pool[target] = pool[source]
    return {"k": s["k"], "v": s["v"]}


# ------------------------------------------------------------------------------------------ the framework's calls
def _plans(tsfm, s):
    """What a program makes once for its cache and its trees: the description of the pages, masks and depths, a workspace."""
    c = s["case"]
    if "plans" not in s:
        s["plans"] = plans = {}
        if c["op"] == "commit":
            plans["pages"] = tsfm.kv_pages(s["k"][0], s["v"][0], s["table"])
            return plans
        plans["pages"] = tsfm.kv_pages(s["k"], s["v"], s["table"])
        size = tsfm.tsfm_tree_attention_workspace(plans["pages"], c["B"], c["M"], c["Hq"], c["longest"])
        plans["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        if c["op"] == "tree":
            n = s["parent"].shape[0]
            plans["mask"] = torch.zeros(n, c["M"], (c["M"] + 63) // 64, dtype=torch.int64, device="cuda")
            plans["depth"] = torch.zeros(n, c["M"], dtype=torch.int32, device="cuda")
            tsfm.tsfm_tree_init(torch.cuda.current_stream().cuda_stream, s["parent"], None, n, c["M"], 0, plans["mask"], plans["depth"])
    return s["plans"]


def _own(s):
    import paper_2511_18191_b200 as tsfm
    c, stream = s["case"], torch.cuda.current_stream().cuda_stream
    if c["op"] == "logprobs":
        x = s["logits"]
        tsfm.tsfm_token_logprobs(stream, x, x.stride(0), c["rows"], c["V"], 1.0 / c["temperature"], s["tokens"] if c["tokens"] else None, c["tokens"],
                                 s["logprob"] if c["tokens"] else None, s["lse"], s["entropy"], c["top"], s["ids"] if c["top"] else None,
                                 s["best"] if c["top"] else None)
        return {k: s[k] for k in ("logprob", "lse", "entropy", "ids", "best")}
    if c["op"] == "verify":
        tsfm.tsfm_verify_tree(stream, s["tokens"], s["parent"], False, s["p"], c["V"], s["q"], c["V"], c["B"], c["M"], c["V"], s["u"], 0, 0, 0,
                              s["n_new"], s["len"], s["out"], s["path"], s["n_accept"], s["len_out"])
        return {"tokens": s["out"], "path": s["path"], "n_accept": s["n_accept"], "len": s["len_out"]}
    plans = _plans(tsfm, s)
    if c["op"] == "commit":
        tsfm.tsfm_cache_commit(stream, plans["pages"], s["path"], s["len"], c["B"], c["M"], c["layers"], s["k"].stride(0))
        return {"k": s["k"], "v": s["v"]}
    if c["op"] == "tree":
        tsfm.tsfm_tree_attention(stream, plans["pages"], s["q"], s["q"].stride(1), s["out"], s["out"].stride(1), s["len"], s["n_new"], plans["mask"],
                                 plans["depth"], c["shared"], c["B"], c["M"], c["Hq"], 1.0 / math.sqrt(c["D"]), c["window"], c["sinks"], c["longest"],
                                 s["lse"], plans["workspace"], plans["workspace"].numel())
    else:
        tsfm.tsfm_window_attention(stream, plans["pages"], s["q"], s["q"].stride(1), s["out"], s["out"].stride(1), s["len"], s["n_new"], c["B"], c["M"],
                                   c["Hq"], 1.0 / math.sqrt(c["D"]), c["window"], c["sinks"], c["longest"], s["lse"], plans["workspace"],
                                   plans["workspace"].numel())
    return {"out": s["out"], "lse": s["lse"]}


def run(s):
    if own:
        return _own(s)
    return {"tree": _run_attend, "window": _run_attend, "logprobs": _run_logprobs, "verify": _run_verify, "commit": _run_commit}[s["case"]["op"]](s)


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(c, seed):
    """From the definitions.  (Nothing of a verification or a commit is a computed number.)"""
    if c["op"] in ("verify", "commit"):
        return None
    s = prepare(c, seed)
    return _exact_logprobs(s, c) if c["op"] == "logprobs" else _exact_attend(s, c)


def _exact_attend(s, c):
    """A series and a key head at a time, all of its slots."""
    Hq, Hkv, D, page = (c[k] for k in ("Hq", "Hkv", "D", "page"))
    G = Hq // Hkv
    out, lse = s["out"].double(), s["lse"].double()
    if sum(_lengths(c)) * Hq * max(_new(c)) * D * 4 > 2e14:
        return None
    for b in range(c["B"]):
        new, length = int(s["n_new"][b]), int(s["len"][b])
        n = length + new
        if not new:
            continue
        slot = torch.arange(n, device="cuda")
        at = s["table"][b].long()[slot // page]
        step = max(1, (1 << 27) // (G * n))
        for m0 in range(0, new, step):
            m = torch.arange(m0, min(new, m0 + step), device="cuda")
            sees = torch.zeros(len(m), n, dtype=torch.bool, device="cuda")
            if c["op"] == "tree":
                row = 0 if c["shared"] else b
                near = slot[:length] - (length + s["depth"][row, m].long())[:, None] > -c["window"] if c["window"] else torch.ones_like(sees[:, :length])
                sees[:, :length] = near | (slot[:length] < c["sinks"])
                sees[:, length:] = s["sees"][row][m, :new]
            else:
                away = (length + m)[:, None] - slot
                sees = (away >= 0) & ((away < c["window"]) | (slot < c["sinks"]))
            lead = torch.zeros_like(sees, dtype=torch.double).masked_fill_(~sees, -math.inf).repeat_interleave(G, 0)
            for h in range(Hkv):
                k, v = (x[at, h, slot % page].double() for x in (s["k"], s["v"]))
                q = s["q"][b, m].double().view(len(m), Hq, D)[:, h * G:(h + 1) * G].reshape(-1, D)
                score = q @ k.T / math.sqrt(D) + lead
                z = torch.logsumexp(score, -1)
                o = torch.exp(score - torch.where(z == -math.inf, torch.zeros_like(z), z)[:, None]) @ v
                out[b, m, h * G * D:(h + 1) * G * D] = o.view(len(m), G * D)
                lse[b, m, h * G:(h + 1) * G] = z.view(len(m), G)
    return {"out": out, "lse": lse}


def _exact_logprobs(s, c):
    rows, V = c["rows"], c["V"]
    out = {"logprob": s["logprob"].double(), "lse": s["lse"].double(), "entropy": s["entropy"].double(), "ids": None,
           "best": torch.full_like(s["best"], -math.inf).double()}
    for r in range(rows):
        x = s["logits"][r].double() / c["temperature"]
        z = torch.logsumexp(x, 0)
        out["lse"][r] = z
        log_p = x - z
        live = log_p[log_p > -math.inf]
        out["entropy"][r] = -(live.exp() * live).sum()
        out["logprob"][r] = log_p[s["tokens"][r].long()]
        if c["top"]:
            out["best"][r, :min(V, c["top"])] = log_p.topk(min(V, c["top"])).values
    return out
