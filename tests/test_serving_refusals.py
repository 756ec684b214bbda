"""Serving over a cache of pages: what the entry points refuse, and their host arithmetic (no GPU needed)."""
import ctypes as C
import math

import pytest

import paper_2511_18191_b200 as tsfm
from tests import serving_ref as ref

ARG, SHAPE = tsfm.TSFM_ERR_ARG, tsfm.TSFM_ERR_SHAPE
A = 1 << 20                                                    # an aligned address that no refused call follows


def pages(**kw):
    p = tsfm.tsfm_kv_pages(A, A, 8 * 16 * 64, 16 * 64, 64, A, 4, 4, 64, 16, 8, 64, tsfm.TSFM_BF16, None)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_PAGES = [(dict(k=None), ARG), (dict(v=None), ARG), (dict(table=None), ARG), (dict(dtype=2), ARG), (dict(n_kv_heads=0), ARG),
             (dict(max_pages=0), ARG), (dict(max_pages=5), ARG), (dict(n_pages=0), ARG), (dict(page_size=0), ARG),
             (dict(page_size=24), SHAPE), (dict(page_size=1 << 17), SHAPE), (dict(d_head=96), SHAPE), (dict(k=A + 8), SHAPE),
             (dict(v=A + 2), SHAPE), (dict(slot_stride=60), SHAPE), (dict(slot_stride=68), SHAPE), (dict(head_stride=1028), SHAPE),
             (dict(page_stride=0), SHAPE), (dict(page_stride=-64), SHAPE)]


def call(fn, **kw):
    """The entry point with good arguments but for `kw`; its code.  Nothing is launched: every case here is refused."""
    pg = kw.pop("pages", pages())
    pg = None if pg is None else C.byref(pg)
    if fn == "append":
        rope = kw.pop("rope", tsfm.tsfm_rope_init(tsfm.TSFM_ROPE_HALF, 64, tsfm.TSFM_ROPE_PLAIN, 1e4))
        d = dict(qkv=A, qs=24 * 64, q_out=A, qos=8 * 64, pos=A, len=A, n_new=A, B=2, M=3, heads=8)
        d.update(kw)
        return tsfm.lib.tsfm_rope_append(None, None if rope is None else C.byref(rope), pg, *d.values())
    if fn == "attend":
        d = dict(q=A, qs=512, out=A, os=512, len=A, n_new=A, B=2, M=3, heads=8, scale=0.1, causal=1, window=0, max_len=64, lse=A,
                 w_in=None, w_out=None, ws=64, work=A, bytes=1 << 40)
        d.update(kw)
        return tsfm.lib.tsfm_paged_attention(None, pg, *d.values())
    if fn == "evict":
        d = dict(dst=A, dst_stride=2, len=A, w=A, ws=64, B=2, budget=32, sinks=4, recent=8, max_len=64, kept=A, w_out=A + 4096, wos=32, len_out=A + 64)
        d.update(kw)
        return tsfm.lib.tsfm_cache_evict(None, pg, *d.values())
    d = dict(tokens=A, p=A, ps=100, q=A, qs=100, B=2, K=4, V=100, u=A, seed=0, rnd=0, s0=0, nd=None, len=A, out=A, n=A, len_out=A)
    d.update(kw)
    return tsfm.lib.tsfm_verify_tokens(None, *d.values())


@pytest.mark.parametrize("fn", ["append", "attend", "evict"])
@pytest.mark.parametrize("change,code", BAD_PAGES + [(None, ARG)])
def test_descriptions_of_pages(fn, change, code):
    assert call(fn, pages=None if change is None else pages(**change)) == code


@pytest.mark.parametrize("fn,change,code", [
    ("append", dict(rope=None), ARG), ("append", dict(qkv=None), ARG), ("append", dict(len=None), ARG), ("append", dict(B=0), ARG),
    ("append", dict(M=0), ARG), ("append", dict(heads=-1), ARG), ("append", dict(heads=0), ARG), ("append", dict(qkv=A + 8), SHAPE),
    ("append", dict(qs=24 * 64 - 8), SHAPE), ("append", dict(qs=24 * 64 + 4), SHAPE), ("append", dict(q_out=A + 4), SHAPE),
    ("append", dict(q_out=A + (1 << 16), qos=8 * 64 - 8), SHAPE), ("append", dict(q_out=A, qos=8 * 64), ARG), ("append", dict(B=1 << 16, M=1 << 16), SHAPE),
    ("append", dict(pages=pages(d_head=32, slot_stride=32)), SHAPE),          # rot_dim 64 beyond the head
    ("attend", dict(q=None), ARG), ("attend", dict(out=None), ARG), ("attend", dict(len=None), ARG), ("attend", dict(work=None), ARG),
    ("attend", dict(window=-1), ARG), ("attend", dict(scale=math.nan), ARG), ("attend", dict(scale=math.inf), ARG), ("attend", dict(w_in=A), ARG),
    ("attend", dict(B=0), ARG), ("attend", dict(M=0), ARG), ("attend", dict(heads=0), ARG), ("attend", dict(max_len=0), ARG),
    ("attend", dict(heads=12), SHAPE), ("attend", dict(q=A + 8), SHAPE), ("attend", dict(out=A + 8), SHAPE), ("attend", dict(qs=504), SHAPE),
    ("attend", dict(os=516), SHAPE), ("attend", dict(w_out=A, ws=63), SHAPE), ("attend", dict(work=A + 128), SHAPE), ("attend", dict(bytes=4096), SHAPE),
    ("attend", dict(max_len=(1 << 30) + 1), SHAPE), ("attend", dict(B=1 << 20, M=1 << 12), SHAPE), ("attend", dict(M=65536, B=1), SHAPE),
    ("evict", dict(dst=None), ARG), ("evict", dict(len=None), ARG), ("evict", dict(w=None), ARG), ("evict", dict(kept=None), ARG),
    ("evict", dict(len_out=None), ARG), ("evict", dict(len_out=A), ARG), ("evict", dict(w_out=A), ARG), ("evict", dict(B=0), ARG),
    ("evict", dict(budget=0), ARG), ("evict", dict(sinks=-1), ARG), ("evict", dict(recent=-1), ARG), ("evict", dict(recent=29), ARG),
    ("evict", dict(max_len=0), ARG), ("evict", dict(ws=63), SHAPE), ("evict", dict(wos=31), SHAPE), ("evict", dict(dst_stride=1), SHAPE),
    ("evict", dict(dst_stride=-1), SHAPE),
    ("verify", dict(p=None), ARG), ("verify", dict(out=None), ARG), ("verify", dict(n=None), ARG), ("verify", dict(tokens=None), ARG),
    ("verify", dict(B=0), ARG), ("verify", dict(K=-1), ARG), ("verify", dict(K=33), ARG), ("verify", dict(V=0), ARG),
    ("verify", dict(V=(1 << 30) + 1, ps=1 << 31, qs=1 << 31), SHAPE), ("verify", dict(ps=99), ARG), ("verify", dict(qs=99), ARG), ("verify", dict(len=None), ARG), ("verify", dict(len_out=None), ARG),
])
def test_arguments(fn, change, code):
    assert call(fn, **change) == code


def test_workspace_sizes():
    size = tsfm.tsfm_paged_attention_workspace
    assert size(pages(), 2, 3, 8, 64) > 0
    # with weights the scores of every row are kept
    assert size(pages(), 2, 3, 8, 1000, True) >= size(pages(), 2, 3, 8, 1000) + 2 * 3 * 8 * 1000 * 4
    # without, it does not grow with the cache
    assert size(pages(), 64, 1, 8, 1 << 17) == size(pages(), 64, 1, 8, 1 << 14)
    for bad in (dict(B=0), dict(M=0), dict(n_heads=9), dict(max_len=0)):
        d = dict(B=2, M=3, n_heads=8, max_len=64)
        d.update(bad)
        assert size(pages(), *d.values()) == 0
    assert size(pages(d_head=80), 2, 3, 8, 64) == 0


@pytest.mark.parametrize("kw", [dict(layout=2), dict(rot=3), dict(rot=-2), dict(rot=130), dict(scaling=4), dict(scaling=-1), dict(base=1.0),
                                dict(base=math.nan), dict(factor=0.5), dict(factor=math.inf), dict(mscale=math.nan),
                                dict(scaling=tsfm.TSFM_ROPE_BASE, rot=2), dict(scaling=tsfm.TSFM_ROPE_PARTS),
                                dict(scaling=tsfm.TSFM_ROPE_PARTS, original=4096.0, lo=4.0, hi=4.0)])
def test_rope_arguments(kw):
    d = dict(layout=0, rot=64, scaling=0, base=1e4, factor=2.0, original=0.0, lo=0.0, hi=0.0, mscale=1.0)
    d.update(kw)
    with pytest.raises(tsfm.TsfmError) as e:
        tsfm.tsfm_rope_init(*d.values())
    assert e.value.code == ARG
    assert tsfm.lib.tsfm_rope_init(None, 0, 64, 0, 1e4, 1.0, 0.0, 0.0, 0.0, 1.0) == ARG


@pytest.mark.parametrize("rot,scaling,name", [(128, 0, "plain"), (64, 1, "linear"), (32, 2, "base"), (64, 3, "parts"), (2, 0, "plain"), (6, 3, "parts")])
def test_rope_frequencies(rot, scaling, name):
    """2^64 times the turns a position: half a unit of 2^-64 turns (a rounding to whole numbers), and the fp64 reference's own few
    roundings of 2^-53."""
    r = tsfm.tsfm_rope_init(0, rot, scaling, 5e5, 8.0, 4096.0, 1.0, 32.0)
    f = ref.frequencies(rot, 5e5, name, 8.0, 4096.0, 1.0, 32.0)
    for i in range(rot // 2):
        assert abs(r.turn[i] / 2.0 ** 64 * 2 * math.pi - f[i]) <= 64 * 2.0 ** -53 * f[i] + math.pi * 2.0 ** -64
    assert all(t == 0 for t in r.turn[rot // 2:])


def test_kv_pages_checks_its_tensors():
    import torch
    k, t = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(3, 4, dtype=torch.int32)
    p = tsfm.kv_pages(k, k.clone(), t)
    assert (p.n_pages, p.n_kv_heads, p.page_size, p.d_head, p.table_stride, p.max_pages) == (4, 2, 16, 64, 4, 4)
    assert (p.page_stride, p.head_stride, p.slot_stride, p.dtype) == (2048, 1024, 64, tsfm.TSFM_BF16)
    n = torch.zeros(4, 16, 2, 64).transpose(1, 2)              # slots before heads
    p = tsfm.kv_pages(n, n, t)
    assert (p.page_stride, p.head_stride, p.slot_stride, p.dtype) == (2048, 64, 128, tsfm.TSFM_F32)
    for bad in [(k.half(), k.half(), t), (k, k.float(), t), (k, k[:3], t), (k, k, t.long()), (k, k, t[0]), (k[..., ::2], k[..., ::2], t),
                (k, torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16).transpose(1, 2), t)]:
        with pytest.raises(tsfm.TsfmError):
            tsfm.kv_pages(*bad)


def test_a_wait_for_a_tile_that_runs_out_is_reported():
    """What no GPU that works can show: the one wait on copies sets the status bit, and both kernels turn their sums into NaN."""
    import os
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_18191_b200", "csrc")
    text = open(os.path.join(csrc, "attn_paged_fetch.cuh")).read()
    uses = [i for i in range(len(text)) if text.startswith("!tile_arrived(", i)]
    assert len(uses) == 1
    after = text[uses[0]:uses[0] + 300]
    assert "dead = true" in after and "sh.dead = 1" in after and "pages_report(a.pg, PAGES_TIMEOUT)" in after
    for f in ("attn_paged_mma.cuh", "attn_paged_f32.cuh"):
        assert "if (TMA && sh.dead)" in open(os.path.join(csrc, f)).read()
