"""Operators of a served model's round over a cache of pages, one call each: rotary positions with the append to the cache,
attention of the new tokens over it, eviction by accumulated attention weight, verification of drafted tokens.

Caches are pools of pages [page, kv head, slot, d_head]; a series' slot s lies in page table[b, s // page_size].  Tables
name pages in no order, and -1 behind a series' last page.  Lengths are spread over a batch by rank (rank**skew of the
longest), so that work(case) follows from the case alone; the seed decides which series has which length.

`own` False computes the operators from elementary torch operations in 32 bits (angles and cumulated probabilities in 64).
"""
import math

import numpy as np
import torch

own = False

F32, BF16 = "f32", "bf16"
TORCH = {F32: torch.float32, BF16: torch.bfloat16}
BYTES = {F32: 4, BF16: 2}


# ------------------------------------------------------------------------------------------ cases
def _append(name, dtype, B, M, Hq, Hkv, D, page, layout, rot, scaling, factor, start, ctx):
    """start: position of the oldest slot still in the cache; ctx: longest length before the append."""
    c = dict(op="append", dtype=dtype, B=B, M=M, Hq=Hq, Hkv=Hkv, D=D, page=page, layout=layout, rot=rot, scaling=scaling,
             factor=factor, start=start, ctx=ctx)
    return dict(c, name=name) if name else c


def _attend(name, dtype, B, M, Hq, Hkv, D, page, longest, skew, window=0, weights=False, causal=True):
    c = dict(op="attend", dtype=dtype, B=B, M=M, Hq=Hq, Hkv=Hkv, D=D, page=page, longest=longest, skew=skew, window=window,
             weights=weights, causal=causal)
    return dict(c, name=name) if name else c


def _evict(name, dtype, B, Hkv, D, page, longest, skew, budget, sinks, recent):
    c = dict(op="evict", dtype=dtype, B=B, Hkv=Hkv, D=D, page=page, longest=longest, skew=skew, budget=budget, sinks=sinks,
             recent=recent)
    return dict(c, name=name) if name else c


def _verify(name, B, K, V, sampled):
    c = dict(op="verify", B=B, K=K, V=V, sampled=sampled)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one series, the smallest models (fp32): latency
        _append("append-one", F32, 1, 1, 4, 4, 32, 16, "half", 32, "plain", 1.0, 0, 30),
        # the K + 1 tokens of a verification pass, ragged, grouped heads, half of each head rotates, long contexts
        _append("append-verification", BF16, 64, 9, 20, 4, 64, 16, "interleaved", 32, "parts", 8.0, 70001, 328),
        # prompts: many tokens at once
        _append("append-prompts", BF16, 16, 2048, 32, 8, 128, 32, "half", 128, "linear", 4.0, 0, 0),
        # one token of one short series, the smallest models (fp32): latency
        _attend("attend-one-short", F32, 1, 1, 4, 4, 32, 16, 31, 0.0),
        # one token of one series with a very long cache: few heads, everything along the length
        _attend("attend-one-long", BF16, 1, 1, 32, 8, 128, 64, 131071, 0.0),
        # a serving batch, one token each, lengths from a few slots to 8192
        _attend("attend-batch", BF16, 256, 1, 32, 8, 128, 32, 8192, 2.0),
        # verification of K = 8 proposals on the 500 M model's heads and capacity
        _attend("attend-verification", BF16, 64, 9, 20, 20, 64, 16, 329, 0.25),
        # grouped heads, several tokens, and the weights that eviction needs
        _attend("attend-weights", BF16, 32, 5, 16, 4, 64, 64, 16001, 1.0, weights=True),
        # one stream that never ends, fp32
        _evict("evict-one", F32, 1, 4, 64, 16, 4100, 0.0, 1024, 4, 128),
        # a batch of them, some short enough to be kept whole
        _evict("evict-batch", BF16, 32, 8, 128, 32, 16384, 1.0, 2048, 4, 512),
        # one series, an ordinary vocabulary: latency
        _verify("verify-one", 1, 4, 32003, True),
        # a batch, a large vocabulary
        _verify("verify-batch", 256, 5, 100003, True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


LARGEST = {"append": 0.8e9, "attend": 2.9e9, "evict": 0.9e9, "verify": 0.2e9}     # bytes of the largest listed cases
DENSE = 256 * 8192 * 8 * 128                                                      # cache elements in a plain form


def _drawn(rng):
    op = rng.choice(["append", "attend", "attend", "evict", "verify"])
    if op == "verify":
        return _verify(None, _log_int(rng, 1, 256), rng.randint(1, 16), _log_int(rng, 100, 131072), rng.random() < 0.75)
    dtype, D, page = rng.choice([F32, BF16, BF16, BF16]), rng.choice([32, 64, 128]), rng.choice([8, 16, 32, 64, 128])
    Hkv = rng.choice([1, 2, 4, 5, 8])
    Hq = Hkv * rng.choice([1, 2, 3, 4, 8])
    if op == "append":
        rot = rng.choice([D, D, D // 2, D // 4, 2 * rng.randint(1, D // 2)])
        scaling = rng.choice(["plain", "linear", "base", "parts"])
        if scaling == "base" and rot == 2:
            scaling = "plain"
        return _append(None, dtype, _log_int(rng, 1, 64), _log_int(rng, 1, 2048), Hq, Hkv, D, page, rng.choice(["half", "interleaved"]), rot,
                       scaling, 1.0 if scaling == "plain" else rng.choice([2.0, 8.0, 32.0]), rng.choice([0, 0, _log_int(rng, 1, 4000000)]), _log_int(rng, 1, 4096))
    B, longest, skew = _log_int(rng, 1, 256), _log_int(rng, 1, 131072), rng.choice([0.0, 0.25, 1.0, 2.0])
    if op == "attend":
        return _attend(None, dtype, B, rng.choice([1, 1, 1, 2, 5, 9, 17]), Hq, Hkv, D, page, longest, skew,
                       window=rng.choice([0, 0, _log_int(rng, 1, longest)]), weights=rng.random() < 0.3, causal=rng.random() < 0.8)
    budget = _log_int(rng, 1, max(1, longest))
    sinks = rng.randint(0, min(8, budget))
    return _evict(None, dtype, B, Hkv, D, page, longest, skew, budget, sinks, rng.randint(0, (budget - sinks) // 2))


def draw(rng):
    while True:
        c = _drawn(rng)
        dense = c["B"] * c["longest"] * c["Hkv"] * c["D"] if "longest" in c else 0
        rows = c["B"] * c["longest"] * c["Hq"] * c["M"] if c["op"] == "attend" else 0
        if work(c)["bytes"] <= LARGEST[c["op"]] and dense <= DENSE and rows <= DENSE // 4:
            return c


def _lengths(c):
    """Slots of each series once the new tokens are in, in ascending order of rank."""
    return [int(round(c["longest"] * ((i + 1) / c["B"]) ** c["skew"])) for i in range(c["B"])]


def _appended(c):
    """(length before, new tokens) of each series, by rank: every fourth one of a batch appends fewer."""
    ctx = [c["ctx"] * (i + 1) // c["B"] for i in range(c["B"])]
    new = [c["M"] if i % 4 != 3 else c["M"] * (i % 7) // 7 for i in range(c["B"])]
    return ctx, new


def work(c):
    if c["op"] == "verify":
        # a row of the target's probabilities a series, one of the draft's where a proposal is rejected
        share = 1.0 - 0.8 ** c["K"] if c["sampled"] else 0.0
        return {"bytes": c["B"] * (c["V"] * 4.0 * (1.0 + share) + c["K"] * 16 + 8), "flops": c["B"] * c["V"] * 2.0}
    e = BYTES[c["dtype"]]
    if c["op"] == "append":
        tokens = sum(_appended(c)[1])
        return {"bytes": tokens * (c["Hq"] + 2 * c["Hkv"]) * c["D"] * 2.0 * e + c["B"] * 12, "flops": tokens * (c["Hq"] + c["Hkv"]) * c["rot"] * 3.0}
    n = _lengths(c)
    if c["op"] == "evict":
        kept = sum(min(x, c["budget"]) for x in n)
        return {"bytes": sum(n) * c["Hkv"] * 4.0 + kept * c["Hkv"] * (4.0 * c["D"] * e + 8), "flops": sum(n) * c["Hkv"] * 1.0}
    M = c["M"]
    span = [min(x, c["window"] + M - 1) if c["window"] else x for x in n]
    new = sum(min(M, x) if c["causal"] else M for x in n)
    rows = [min(M, x) if c["causal"] else M for x in n]
    b = sum(span) * c["Hkv"] * c["D"] * 2.0 * e + new * c["Hq"] * (2.0 * c["D"] * e + 4) + (sum(n) * c["Hkv"] * 8.0 if c["weights"] else 0.0)
    return {"bytes": b + c["B"] * 8, "flops": sum(r * s for r, s in zip(rows, span)) * c["Hq"] * 4.0 * c["D"]}


# ------------------------------------------------------------------------------------------ inputs
def _int(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _pages(c, slots, order, spare=0):
    """A table [B, most pages] for series of `slots` slots each, the pages in a shuffled order, and the pool's size."""
    page = c["page"]
    counts = [-(-s // page) for s in slots]
    most, total = max(1, max(counts)), sum(counts) + spare
    perm = order.permutation(total).astype(np.int32)
    table = np.full((len(slots), most), -1, np.int32)
    at = 0
    for row, k in zip(table, counts):
        row[:k] = perm[at:at + k]
        at += k
    return torch.from_numpy(table).cuda(), total, perm[at:]


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    order = np.random.RandomState(seed % (1 << 32))
    s = {"case": c}
    if c["op"] == "verify":
        return _prepare_verify(s, c, g)
    t, B, Hkv, D = TORCH[c["dtype"]], c["B"], c["Hkv"], c["D"]

    def normal(*shape):
        x = torch.empty(shape, dtype=t, device="cuda")
        return x.normal_(generator=g)

    which = order.permutation(B)
    if c["op"] == "append":
        ctx, new = ([v[i] for i in which] for v in _appended(c))
        M, Hq = c["M"], c["Hq"]
        s["len"], s["n_new"], s["pos"] = _int(ctx), _int(new), _int([x + c["start"] for x in ctx])
        s["table"], n, _ = _pages(c, [x + M for x in ctx], order)
        s["qkv"] = normal(B, M, (Hq + 2 * Hkv) * D)
        s["q_out"] = torch.zeros(B, M, Hq * D, dtype=t, device="cuda")
        s["k"], s["v"] = (torch.zeros(n, Hkv, c["page"], D, dtype=t, device="cuda") for _ in "kv")
        return s
    total = [_lengths(c)[i] for i in which]
    if c["op"] == "attend":
        M, Hq = c["M"], c["Hq"]
        s["table"], n, _ = _pages(c, total, order)
        new = [min(M, x) if c["causal"] else M for x in total]
        s["n_new"], s["len"] = _int(new), _int([x - y if c["causal"] else x for x, y in zip(total, new)])
        s["k"], s["v"] = (normal(max(1, n), Hkv, c["page"], D) for _ in "kv")
        s["q"] = normal(B, M, Hq * D) * 2               # scores of standard deviation 2: neither flat nor one slot
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(B, M, Hq, device="cuda")
        if c["weights"]:
            s["w"] = torch.rand(B, Hkv, c["longest"], generator=g, device="cuda")
            s["w_out"] = torch.zeros_like(s["w"])
        return s
    s["len"] = _int(total)
    s["table"], n, _ = _pages(c, total, order)
    s["dst_table"], m, _ = _pages(c, [min(x, c["budget"]) for x in total], order)
    s["dst_table"] = torch.where(s["dst_table"] >= 0, s["dst_table"] + n, s["dst_table"])
    s["k"], s["v"] = (normal(max(1, n + m), Hkv, c["page"], D) for _ in "kv")
    # accumulated weights are heavy-tailed, and exactly 0 where a window has long passed
    w = torch.rand(B, Hkv, c["longest"], generator=g, device="cuda")
    s["w"] = torch.where(w < 0.1, torch.zeros_like(w), (1.0 - w).log().square())
    s["w_out"] = torch.zeros(B, Hkv, c["budget"], device="cuda")
    s["kept"] = torch.full((B, Hkv, c["budget"]), -2, dtype=torch.int32, device="cuda")
    s["len_out"] = torch.zeros_like(s["len"])
    return s


def _prepare_verify(s, c, g):
    B, K, V = c["B"], c["K"], c["V"]
    # a draft that tracks its target, both cut to their likelier tokens as samplers do
    x = torch.randn(B, K + 1, V, generator=g, device="cuda") * 2.5

    def probabilities(x):
        p = torch.softmax(x, -1)
        p = torch.where(p < 0.02 / V, torch.zeros_like(p), p)
        return p / p.sum(-1, keepdim=True)

    q = probabilities(x[:, :K])
    s["p"] = probabilities(x + 0.5 * torch.randn(x.shape, generator=g, device="cuda"))
    s["tokens"] = (torch.multinomial(q.view(-1, V), 1, generator=g) if c["sampled"] else q.view(-1, V).argmax(-1)).view(B, K).int()
    s["q"] = q if c["sampled"] else None
    s["u"] = torch.rand(B, K + 1, generator=g, device="cuda")
    s["len"] = torch.randint(1, 5000, (B,), generator=g, device="cuda", dtype=torch.int32)
    s["out"] = torch.zeros(B, K + 1, dtype=torch.int32, device="cuda")
    s["n_accept"], s["len_out"] = torch.zeros_like(s["len"]), torch.zeros_like(s["len"])
    return s


# ------------------------------------------------------------------------------------------ plain forms
ORIGINAL, TURNS_LO, TURNS_HI, BASE = 4096.0, 1.0, 32.0, 10000.0      # of "parts"; base of all


def _mscale(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "parts" else 1.0


def _frequencies(c):
    rot, F = c["rot"], c["factor"]
    i = torch.arange(0, rot, 2, device="cuda", dtype=torch.float64)
    if c["scaling"] == "base":
        return (BASE * F ** (rot / (rot - 2.0))) ** (-i / rot)
    f = BASE ** (-i / rot)
    if c["scaling"] == "linear":
        return f / F
    if c["scaling"] == "parts":
        ramp = ((ORIGINAL * f / (2 * math.pi) - TURNS_LO) / (TURNS_HI - TURNS_LO)).clamp(0, 1)
        return f * (ramp + (1 - ramp) / F)
    return f


def _rotate(x, cos, sin, c):
    """x [B, M, heads, D] in 32 bits."""
    r = c["rot"]
    if c["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _run_append(s):
    c = s["case"]
    B, M, Hq, Hkv, D, page = (c[k] for k in ("B", "M", "Hq", "Hkv", "D", "page"))
    m = torch.arange(M, device="cuda")
    angle = (s["pos"][:, None] + m).double()[..., None] * _frequencies(c)
    cos, sin = ((f(angle) * _mscale(c)).float()[:, :, None] for f in (torch.cos, torch.sin))
    x = s["qkv"].float().view(B, M, Hq + 2 * Hkv, D)
    live = m < s["n_new"][:, None]
    turned = _rotate(x[:, :, :Hq + Hkv], cos, sin, c).to(s["qkv"].dtype)
    q_out = torch.where(live[..., None], turned[:, :, :Hq].reshape(B, M, Hq * D), s["q_out"])
    b, t = live.nonzero(as_tuple=True)
    slot = s["len"][b].long() + t
    at = (s["table"][b, slot // page].long(), slice(None), slot % page)
    s["k"][at] = turned[b, t, Hq:]
    s["v"][at] = x[b, t, Hq + Hkv:].to(s["v"].dtype)
    return {"q": q_out, "k": s["k"], "v": s["v"]}


def _dense(pool, table, L):
    """[B, kv heads, L, D] in 32 bits."""
    B, _, page, D = table.shape[0], *pool.shape[1:]
    x = pool[table[:, :-(-L // page)].clamp(min=0).long()].transpose(1, 2)
    return x.reshape(B, pool.shape[1], -1, D)[:, :, :L].float()


def _run_attend(s):
    c = s["case"]
    B, M, Hq, Hkv, D, L = (c[k] for k in ("B", "M", "Hq", "Hkv", "D", "longest"))
    G = Hq // Hkv
    m, slot = torch.arange(M, device="cuda"), torch.arange(L, device="cuda")
    end = (s["len"][:, None] + m + 1) if c["causal"] else s["len"][:, None].expand(B, M)
    seen = slot < end[..., None]
    if c["window"]:
        seen = seen & (slot >= end[..., None] - c["window"])
    live = m < s["n_new"][:, None]
    k, v = _dense(s["k"], s["table"], L), _dense(s["v"], s["table"], L)
    gone = ~(seen & live[..., None]).any(1)[:, None, :, None]
    k, v = k.masked_fill_(gone, 0.0), v.masked_fill_(gone, 0.0)
    q = s["q"].float().view(B, M, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, M * G, D)
    score = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    hidden = ~seen[:, None, :, None].expand(B, Hkv, M, G, L).reshape(B, Hkv, M * G, L)
    score = score.masked_fill_(hidden, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = (score - top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    o = torch.matmul(p, v).view(B, Hkv, M, G, D).permute(0, 2, 1, 3, 4).reshape(B, M, Hq * D)
    lse = (top + total.log()).view(B, Hkv, M, G).permute(0, 2, 1, 3).reshape(B, M, Hq)
    out = {"out": torch.where(live[..., None], o.to(s["out"].dtype), s["out"]), "lse": torch.where(live[..., None], lse, s["lse"])}
    if c["weights"]:
        p = p.masked_fill_(~live[:, None, :, None].expand(B, Hkv, M, G).reshape(B, Hkv, M * G, 1), 0.0)
        ends = s["len"] + s["n_new"] if c["causal"] else s["len"]
        out["w"] = torch.where((slot < ends[:, None])[:, None], s["w"] + p.sum(2), s["w_out"])
    return out


def _run_evict(s):
    c = s["case"]
    B, Hkv, D, page, L, budget = (c[k] for k in ("B", "Hkv", "D", "page", "longest", "budget"))
    n = s["len"].long()[:, None, None]
    slot = torch.arange(L, device="cuda").expand(B, Hkv, L)
    forced = (slot < c["sinks"]) | (slot >= n - c["recent"]) | (n <= budget)
    key = torch.where(forced, torch.full_like(s["w"], math.inf), s["w"]).masked_fill_(slot >= n, -math.inf)
    best = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :budget]
    count = n.clamp(max=budget)
    j = torch.arange(min(budget, L), device="cuda")
    kept = torch.sort(torch.where(j < count, best, torch.full_like(best, L)), dim=-1).values
    live = (j < count) & (kept < L)
    kept = torch.where(live, kept, torch.full_like(kept, -1))
    s["kept"].fill_(-1)
    s["kept"][..., :kept.shape[-1]] = kept.int()
    s["w_out"][..., :kept.shape[-1]] = torch.where(live, s["w"].gather(-1, kept.clamp(min=0)), s["w_out"][..., :kept.shape[-1]])
    b, h, j = live.nonzero(as_tuple=True)
    old = kept[b, h, j]
    source = (s["table"][b, old // page].long(), h, old % page)
    target = (s["dst_table"][b, j // page].long(), h, j % page)
    for pool in (s["k"], s["v"]):
        pool[target] = pool[source]
    s["len_out"].copy_(s["len"].clamp(max=budget))
    return {"kept": s["kept"], "w": s["w_out"], "len": s["len_out"], "k": s["k"], "v": s["v"]}


def _run_verify(s):
    c = s["case"]
    B, K, V = c["B"], c["K"], c["V"]
    tokens, i = s["tokens"].long(), torch.arange(K + 1, device="cuda")
    px = s["p"][:, :K].gather(2, tokens[..., None])[..., 0].double()
    qx = s["q"].gather(2, tokens[..., None])[..., 0].double() if c["sampled"] else torch.ones_like(px)
    n = (s["u"][:, :K].double() * qx < px).int().cumprod(1).sum(1)
    b = torch.arange(B, device="cuda")
    p = s["p"][b, n].double()
    rejected = n.clamp(max=K - 1)
    if c["sampled"]:
        q = s["q"][b, rejected].double()
    else:
        q = torch.zeros_like(p).scatter_(1, tokens[b, rejected][:, None], 1.0)
    rest = torch.where((n < K)[:, None], (p - q).clamp(min=0), p)
    rest = torch.where(rest.sum(1, keepdim=True) > 0, rest, p)
    cdf = rest.cumsum(1)
    t = (cdf <= s["u"][:, K:].double() * cdf[:, -1:]).sum(1)
    t = torch.minimum(t, V - 1 - (rest.flip(1) > 0).int().argmax(1))
    drafted = torch.cat([tokens, torch.full((B, 1), -1, dtype=torch.long, device="cuda")], 1)
    out = torch.where(i < n[:, None], drafted, torch.where(i == n[:, None], t[:, None], torch.full_like(drafted, -1)))
    return {"tokens": out.int(), "n_accept": n.int(), "len": (s["len"] + n + 1).int()}


# ------------------------------------------------------------------------------------------ the framework's calls
def _plans(tsfm, s):
    """What a program makes once for its cache and model: the description of the pages, the frequencies, a workspace."""
    c = s["case"]
    if "plans" not in s:
        s["plans"] = {"pages": tsfm.kv_pages(s["k"], s["v"], s["table"])}
        if c["op"] == "append":
            s["plans"]["rope"] = tsfm.tsfm_rope_init(
                tsfm.TSFM_ROPE_HALF if c["layout"] == "half" else tsfm.TSFM_ROPE_INTERLEAVED, c["rot"],
                {"plain": tsfm.TSFM_ROPE_PLAIN, "linear": tsfm.TSFM_ROPE_LINEAR, "base": tsfm.TSFM_ROPE_BASE, "parts": tsfm.TSFM_ROPE_PARTS}[c["scaling"]],
                BASE, c["factor"], ORIGINAL, TURNS_LO, TURNS_HI, _mscale(c))
        if c["op"] == "attend":
            size = tsfm.tsfm_paged_attention_workspace(s["plans"]["pages"], c["B"], c["M"], c["Hq"], c["longest"], c["weights"])
            s["plans"]["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s["plans"]


def _own(s):
    import paper_2511_18191_b200 as tsfm
    c, stream = s["case"], torch.cuda.current_stream().cuda_stream
    if c["op"] == "verify":
        tsfm.tsfm_verify_tokens(stream, s["tokens"], s["p"], c["V"], s["q"], c["V"], c["B"], c["K"], c["V"], s["u"], 0, 0, 0,
                                None, s["len"], s["out"], s["n_accept"], s["len_out"])
        return {"tokens": s["out"], "n_accept": s["n_accept"], "len": s["len_out"]}
    plans = _plans(tsfm, s)
    if c["op"] == "append":
        tsfm.tsfm_rope_append(stream, plans["rope"], plans["pages"], s["qkv"], s["qkv"].stride(1), s["q_out"], s["q_out"].stride(1),
                              s["pos"], s["len"], s["n_new"], c["B"], c["M"], c["Hq"])
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    if c["op"] == "attend":
        w, w_out = (s["w"], s["w_out"]) if c["weights"] else (None, None)
        tsfm.tsfm_paged_attention(stream, plans["pages"], s["q"], s["q"].stride(1), s["out"], s["out"].stride(1), s["len"], s["n_new"],
                                  c["B"], c["M"], c["Hq"], 1.0 / math.sqrt(c["D"]), c["causal"], c["window"], c["longest"], s["lse"],
                                  w, w_out, c["longest"], plans["workspace"], plans["workspace"].numel())
        return {"out": s["out"], "lse": s["lse"], **({"w": w_out} if c["weights"] else {})}
    tsfm.tsfm_cache_evict(stream, plans["pages"], s["dst_table"], s["dst_table"].shape[1], s["len"], s["w"], c["longest"], c["B"],
                          c["budget"], c["sinks"], c["recent"], c["longest"], s["kept"], s["w_out"], c["budget"], s["len_out"])
    return {"kept": s["kept"], "w": s["w_out"], "len": s["len_out"], "k": s["k"], "v": s["v"]}


def run(s):
    if own:
        return _own(s)
    return {"append": _run_append, "attend": _run_attend, "evict": _run_evict, "verify": _run_verify}[s["case"]["op"]](s)


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(c, seed):
    """From the definitions, series by series.  (Nothing of a verification is a computed number.)"""
    if c["op"] == "verify":
        return None
    s = prepare(c, seed)
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict}[c["op"]](s, c)


def _where(s, b, slots, page, table="table"):
    return s[table][b].long()[slots // page], slots % page


def _exact_append(s, c):
    B, M, Hq, Hkv, D, page, rot = (c[k] for k in ("B", "M", "Hq", "Hkv", "D", "page", "rot"))
    pairs = []
    for i in range(rot // 2):
        f = BASE ** (-2.0 * i / rot)
        if c["scaling"] == "linear":
            f /= c["factor"]
        elif c["scaling"] == "base":
            f = (BASE * c["factor"] ** (rot / (rot - 2.0))) ** (-2.0 * i / rot)
        elif c["scaling"] == "parts":
            turns = ORIGINAL * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - TURNS_LO) / (TURNS_HI - TURNS_LO)))
            f *= keep + (1.0 - keep) / c["factor"]
        pairs.append((i, i + rot // 2, f) if c["layout"] == "half" else (2 * i, 2 * i + 1, f))
    first, second = ([p[k] for p in pairs] for k in (0, 1))
    f = torch.tensor([p[2] for p in pairs], dtype=torch.float64, device="cuda")
    q_out, k, v = s["q_out"].double(), s["k"].double(), s["v"].double()
    for b in range(B):
        new, length, pos = int(s["n_new"][b]), int(s["len"][b]), int(s["pos"][b])
        x = s["qkv"][b, :new].double().view(new, Hq + 2 * Hkv, D)
        z = torch.polar(torch.full((new, len(pairs)), _mscale(c), dtype=torch.float64, device="cuda"), torch.arange(pos, pos + new, device="cuda").double()[:, None] * f)
        turned = torch.complex(x[:, :Hq + Hkv, first], x[:, :Hq + Hkv, second]) * z[:, None]
        x[:, :Hq + Hkv, first], x[:, :Hq + Hkv, second] = turned.real, turned.imag
        q_out[b, :new] = x[:, :Hq].reshape(new, Hq * D)
        at, slot = _where(s, b, torch.arange(length, length + new, device="cuda"), page)
        k[at, :, slot], v[at, :, slot] = x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    return {"q": q_out, "k": k, "v": v}


def _exact_attend(s, c):
    B, M, Hq, Hkv, D, page = (c[k] for k in ("B", "M", "Hq", "Hkv", "D", "page"))
    G = Hq // Hkv
    out, lse = s["out"].double(), s["lse"].double()
    w = s["w_out"].double() if c["weights"] else None
    for b in range(B):
        new, length = int(s["n_new"][b]), int(s["len"][b])
        n = length + new if c["causal"] else length
        at, slot = _where(s, b, torch.arange(n, device="cuda"), page)
        k, v = s["k"][at, :, slot].double(), s["v"][at, :, slot].double()             # [n, Hkv, D]
        got = torch.zeros(Hkv, n, dtype=torch.float64, device="cuda")
        for m in range(new):
            end = length + m + 1 if c["causal"] else length
            start = max(0, end - c["window"]) if c["window"] else 0
            if end <= start:
                out[b, m], lse[b, m] = 0.0, -math.inf
                continue
            q = s["q"][b, m].double().view(Hkv, G, D)
            score = torch.einsum("hgd,nhd->hgn", q, k[start:end]) / math.sqrt(D)
            z = torch.logsumexp(score, -1)
            p = torch.exp(score - z[..., None])
            out[b, m], lse[b, m] = torch.einsum("hgn,nhd->hgd", p, v[start:end]).reshape(-1), z.reshape(-1)
            got[:, start:end] += p.sum(1)
        if w is not None:
            w[b, :, :n] = s["w"][b, :, :n].double() + got
    return {"out": out, "lse": lse, **({"w": w} if c["weights"] else {})}


def _exact_evict(s, c):
    w, length = s["w"].cpu().numpy(), s["len"].tolist()
    got = s["w_out"].double().cpu()
    for b, n in enumerate(length):
        for h in range(c["Hkv"]):
            if n <= c["budget"]:
                kept = np.arange(n)
            else:
                middle = np.arange(c["sinks"], n - c["recent"])
                best = middle[np.lexsort((middle, -w[b, h, middle].astype(np.float64)))][:c["budget"] - c["sinks"] - c["recent"]]
                kept = np.sort(np.concatenate([np.arange(c["sinks"]), best, np.arange(n - c["recent"], n)]))
            got[b, h, :len(kept)] = torch.from_numpy(w[b, h, kept].astype(np.float64))
    return {"kept": None, "w": got, "len": None, "k": None, "v": None}
