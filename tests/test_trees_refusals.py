"""Trees, windows with sinks, log probabilities: what the entry points refuse, and their host arithmetic (no GPU needed)."""
import ctypes as C
import math

import pytest

import paper_2511_18191_b200 as tsfm
from tests.test_serving_refusals import A, ARG, BAD_PAGES, SHAPE, pages


def call(fn, **kw):
    """The entry point with good arguments but for `kw`; its code.  Nothing is launched: every case here is refused."""
    pg = kw.pop("pages", pages())
    pg = None if pg is None else C.byref(pg)
    lib = tsfm.lib
    if fn == "init":
        d = dict(parent=A, n_new=A, B=2, M=7, window=0, mask=A, depth=A)
        d.update(kw)
        return lib.tsfm_tree_init(None, *d.values())
    if fn == "append":
        d = dict(qkv=A, qs=24 * 64, q_out=A, qos=24 * 64, pos=A, len=A, n_new=A, depth=A, shared=0, B=2, M=3, heads=8)
        d.update(kw)
        rope = tsfm.tsfm_rope_init(tsfm.TSFM_ROPE_HALF, 64, tsfm.TSFM_ROPE_PLAIN, 1e4)
        return lib.tsfm_rope_append_tree(None, C.byref(rope), pg, *d.values())
    if fn == "tree":
        d = dict(q=A, qs=512, out=A, os=512, len=A, n_new=A, mask=A, depth=A, shared=0, B=2, M=3, heads=8, scale=0.1, window=0, sinks=0, max_len=64,
                 lse=A, work=A, bytes=1 << 40)
        d.update(kw)
        return lib.tsfm_tree_attention(None, pg, *d.values())
    if fn == "window":
        d = dict(q=A, qs=512, out=A, os=512, len=A, n_new=A, B=2, M=3, heads=8, scale=0.1, window=9, sinks=4, max_len=64, lse=A, work=A, bytes=1 << 40)
        d.update(kw)
        return lib.tsfm_window_attention(None, pg, *d.values())
    if fn == "logprobs":
        d = dict(x=A, stride=100, dtype=tsfm.TSFM_BF16, rows=3, V=100, scale=1.0, tokens=A, n_tokens=1, logprob=A, lse=A, entropy=A, n_top=5, ids=A, best=A)
        d.update(kw)
        return lib.tsfm_token_logprobs(None, *d.values())
    if fn == "verify":
        d = dict(tokens=A, parent=A, shared=0, p=A, ps=100, q=A, qs=100, B=2, M=4, V=100, u=A, seed=0, rnd=0, s0=0, n_new=None, len=A, out=A, path=A, n=A,
                 len_out=A)
        d.update(kw)
        return lib.tsfm_verify_tree(None, *d.values())
    d = dict(path=A, len=A, B=2, M=4, layers=1, stride=0)
    d.update(kw)
    return lib.tsfm_cache_commit(None, pg, *d.values())


@pytest.mark.parametrize("fn", ["append", "tree", "window", "commit"])
@pytest.mark.parametrize("change,code", BAD_PAGES + [(None, ARG)])
def test_descriptions_of_pages(fn, change, code):
    assert call(fn, pages=None if change is None else pages(**change)) == code


ATTENTION = [(dict(q=None), ARG), (dict(out=None), ARG), (dict(len=None), ARG), (dict(work=None), ARG), (dict(window=-1), ARG), (dict(sinks=-1), ARG),
             (dict(scale=math.nan), ARG), (dict(scale=math.inf), ARG), (dict(scale=3e38), ARG), (dict(B=0), ARG), (dict(M=0), ARG), (dict(heads=0), ARG),
             (dict(max_len=0), ARG), (dict(heads=12), SHAPE), (dict(q=A + 8), SHAPE), (dict(out=A + 8), SHAPE), (dict(qs=504), SHAPE), (dict(os=516), SHAPE),
             (dict(work=A + 128), SHAPE), (dict(bytes=4096), SHAPE), (dict(max_len=(1 << 30) + 1), SHAPE)]


@pytest.mark.parametrize("fn,change,code", [(f, c, code) for f in ("tree", "window") for c, code in ATTENTION] + [
    ("tree", dict(mask=None), ARG), ("tree", dict(window=5, depth=None), ARG), ("tree", dict(M=257), SHAPE),
    ("window", dict(M=65536, B=1), SHAPE), ("window", dict(B=1 << 20, M=1 << 12), SHAPE),
    ("init", dict(parent=None), ARG), ("init", dict(mask=None), ARG), ("init", dict(depth=None), ARG), ("init", dict(B=0), ARG), ("init", dict(M=0), ARG),
    ("init", dict(window=-1), ARG), ("init", dict(M=257), SHAPE),
    ("append", dict(depth=None), ARG), ("append", dict(qkv=None), ARG), ("append", dict(q_out=A + 4), SHAPE), ("append", dict(qos=8 * 64), ARG),
    ("logprobs", dict(x=None), ARG), ("logprobs", dict(dtype=2), ARG), ("logprobs", dict(rows=0), ARG), ("logprobs", dict(V=0), ARG),
    ("logprobs", dict(stride=99), ARG), ("logprobs", dict(scale=0.0), ARG), ("logprobs", dict(scale=-1.0), ARG), ("logprobs", dict(scale=math.nan), ARG),
    ("logprobs", dict(scale=math.inf), ARG), ("logprobs", dict(scale=3e38), ARG), ("logprobs", dict(tokens=None), ARG), ("logprobs", dict(logprob=None), ARG),
    ("logprobs", dict(n_tokens=-1), ARG), ("logprobs", dict(n_top=-1), ARG), ("logprobs", dict(ids=None), ARG), ("logprobs", dict(best=None), ARG),
    ("logprobs", dict(n_top=33), SHAPE), ("logprobs", dict(x=A + 1), SHAPE), ("logprobs", dict(V=(1 << 30) + 1, stride=1 << 31), SHAPE),
    ("verify", dict(tokens=None), ARG), ("verify", dict(parent=None), ARG), ("verify", dict(p=None), ARG), ("verify", dict(out=None), ARG),
    ("verify", dict(path=None), ARG), ("verify", dict(n=None), ARG), ("verify", dict(B=0), ARG), ("verify", dict(M=0), ARG), ("verify", dict(V=0), ARG),
    ("verify", dict(M=257), SHAPE), ("verify", dict(V=(1 << 30) + 1, ps=1 << 31, qs=1 << 31), SHAPE), ("verify", dict(ps=99), ARG),
    ("verify", dict(qs=99), ARG), ("verify", dict(len=None), ARG), ("verify", dict(len_out=None), ARG),
    ("commit", dict(path=None), ARG), ("commit", dict(len=None), ARG), ("commit", dict(B=0), ARG), ("commit", dict(M=0), ARG), ("commit", dict(layers=0), ARG),
    ("commit", dict(M=257), SHAPE), ("commit", dict(layers=2, stride=0), SHAPE), ("commit", dict(layers=2, stride=8196), SHAPE),
    ("commit", dict(layers=2, stride=-8192), SHAPE),
])
def test_arguments(fn, change, code):
    assert call(fn, **change) == code


def test_workspace_sizes():
    size = tsfm.tsfm_tree_attention_workspace
    assert size(pages(), 2, 3, 8, 64) > 0
    # it does not grow with the cache, nor without limit with the tokens
    assert size(pages(), 64, 16, 8, 1 << 17) == size(pages(), 64, 16, 8, 1 << 14)
    assert size(pages(), 64, 4096, 8, 1 << 14) <= 2 * size(pages(), 64, 256, 8, 1 << 14)
    for bad in (dict(B=0), dict(M=0), dict(n_heads=9), dict(max_len=0), dict(M=65536)):
        d = dict(B=2, M=3, n_heads=8, max_len=64)
        d.update(bad)
        assert size(pages(), *d.values()) == 0
    assert size(pages(d_head=80), 2, 3, 8, 64) == 0


def test_the_binding_refuses_tensors_that_the_library_would_misread():
    import torch
    x = torch.zeros(4, dtype=torch.int32)                      # on the host
    for f in (lambda: tsfm.tsfm_tree_init(0, x, None, 1, 4, 0, x, x), lambda: tsfm.tsfm_cache_commit(0, pages(), x, x, 1, 4),
              lambda: tsfm.tsfm_token_logprobs(0, x.float(), 4, 1, 4, 1.0, None, 0, None, None, None, 0, None, None),
              lambda: tsfm.tsfm_verify_tree(0, x, x, False, x.float(), 1, None, 0, 1, 4, 1, None, 0, 0, 0, None, None, x, x, x, None)):
        with pytest.raises(tsfm.TsfmError) as e:
            f()
        assert e.value.code == ARG
