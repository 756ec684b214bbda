"""Serving over a cache of pages, at the edges of what a call may be given: what needs no GPU."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_2511_18191_b200 as tsfm
from tests.test_serving_refusals import A, ARG, SHAPE, call, pages

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WALK = r"""
#include <cstdio>
#include <vector>
#include "attn_paged.cuh"
using namespace tsfm;
// The walk from tile `first` of series b0 over `count` tiles; spans as they are now, `later` as they are once the walk has begun.
static int walk(const std::vector<int> &now, const std::vector<int> &later, int units, int b0, int count, bool print) {
  int b = b0, u = 0, t = 0, calls = 0;
  PagedSpan sp{};
  sp.tiles = now[b];
  for (int i = 0; i < count; ++i) {
    if (print) std::printf("%d %d %d\n", b, u, t);
    if (b < 0 || b >= (int)now.size() || u < 0 || u >= units || t < 0 || calls > (int)now.size()) return 1;
    if (i + 1 < count)
      paged_next_tile(b, u, t, sp, (int)now.size(), units, [&]() {
        ++calls;
        PagedSpan s{};
        s.tiles = later[b];
        return s;
      });
  }
  return 0;
}
int main() {
  const std::vector<int> lengths = {0, 2, 0, 0, 1, 3, 0}, none(7, 0), long_ones(7, 1 << 20);
  if (walk(lengths, lengths, 2, 1, 2 * (2 + 1 + 3), true)) return 2;
  for (int b0 : {1, 4, 5})
    for (const auto &later : {none, long_ones, std::vector<int>{0, 0, 0, 1, 0, 0, 0}})
      if (walk(lengths, later, 2, b0, 1000, false)) return 3;
  return 0;
}
"""


@pytest.mark.skipif(shutil.which(os.environ.get("NVCC", "nvcc")) is None, reason="no nvcc")
def test_the_walk_over_tiles_ends_whatever_lengths_become(tmp_path):
    """Every unit's tiles in order, empty series left out; and where lengths are others than at the start (a call that overlaps another one
    that writes them), no more steps than series, and no index outside."""
    src, exe = tmp_path / "walk.cu", tmp_path / "walk"
    src.write_text(WALK)
    subprocess.run([os.environ.get("NVCC", "nvcc"), "-std=c++17", "-O1", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2511_18191_b200", "csrc"), "-o", str(exe), str(src)], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    want = [(b, u, t) for b, n in ((1, 2), (4, 1), (5, 3)) for u in range(2) for t in range(n)]
    assert run.returncode == 0 and [tuple(map(int, x.split())) for x in run.stdout.splitlines()] == want


@pytest.mark.parametrize("dtype", [tsfm.TSFM_F32, tsfm.TSFM_BF16])
@pytest.mark.parametrize("heads,kv", [(1 << 25, 8), (1 << 24, 8), (8, 1 << 24), (2 ** 31 - 1, 8), (0, 2 ** 31 - 1)])
def test_rows_of_an_append_stay_below_32_bits(dtype, heads, kv):
    """2^25 heads of 64 are 2^31 elements: their places within a row would not fit the kernels' 32-bit offsets (the limit is half of that, so that
    no loop over a row passes them either)."""
    assert call("append", pages=pages(dtype=dtype, n_kv_heads=kv), heads=heads, qs=1 << 40, q_out=None) == SHAPE


@pytest.mark.parametrize("B,M,heads,max_len", [(1 << 20, 2047, 32, 1 << 30), (1 << 16, 1000, 64, 1 << 30), (1 << 20, 1, 8, 1 << 30)])
def test_workspaces_that_no_memory_holds(B, M, heads, max_len):
    """The scores of these shapes take 2^64 bytes and more (the size would come out small), or 2^55."""
    kv = pages(n_kv_heads=1)
    assert tsfm.tsfm_paged_attention_workspace(kv, B, M, heads, max_len, True) == 0
    assert tsfm.tsfm_paged_attention_workspace(kv, B, M, heads, max_len, False) > 0       # without weights there are none
    assert call("attend", pages=kv, B=B, M=M, heads=heads, max_len=max_len, w_out=A, ws=max_len, qs=heads * 64, os=heads * 64, bytes=2 ** 64 - 1) == SHAPE


@pytest.mark.parametrize("scale", [2.4e38, -2.4e38, 3.4e38])
def test_a_scale_that_base_2_does_not_hold(scale):
    """scale * log2(e) beyond the largest float: a score of 0 would become 0 x inf."""
    assert call("attend", scale=scale) == ARG


class Fake:
    """What the binding looks at of a tensor, on a device that need not exist."""

    def __init__(self, dtype, device=0, contiguous=True):
        self.dtype, self.device, self.contiguous = dtype, device, contiguous

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return A


I32, F32, BF16 = torch.int32, torch.float32, torch.bfloat16
# arguments of each call in order; tensors by their types, (type,) where the call reads them as contiguous
CALLS = {
    "append": ("tsfm_rope_append", dict(stream=None, rope=None, pages=None, qkv=BF16, qs=24 * 64, q_out=BF16, qos=8 * 64, pos=(I32,), len=(I32,), n_new=(I32,),
                                        B=2, M=3, heads=8)),
    "attend": ("tsfm_paged_attention", dict(stream=None, pages=None, q=BF16, qs=512, out=BF16, os=512, len=(I32,), n_new=(I32,), B=2, M=3, heads=8, scale=0.1,
                                            causal=True, window=0, max_len=64, lse=(F32,), w_in=F32, w_out=F32, ws=64, work=(torch.uint8,), bytes=1)),
    "evict": ("tsfm_cache_evict", dict(stream=None, pages=None, dst=I32, ds=2, len=(I32,), w=F32, ws=64, B=2, budget=32, sinks=4, recent=8, max_len=64,
                                       kept=(I32,), w_out=F32, wos=32, len_out=(I32,))),
    "verify": ("tsfm_verify_tokens", dict(stream=None, tokens=(I32,), p=F32, ps=100, q=F32, qs=100, B=2, K=4, V=100, u=(F32,), seed=0, rnd=0, s0=0, nd=(I32,),
                                          len=(I32,), out=(I32,), n=(I32,), len_out=(I32,))),
}
TENSORS = [(fn, name, kind) for fn, (_, args) in CALLS.items() for name, kind in args.items() if isinstance(kind, (tuple, torch.dtype))]


def through_the_binding(monkeypatch, fn, **change):
    """The call with tensors as it wants them but for `change`; the code that comes back, 0 where it reached the library (a stand-in)."""
    from paper_2511_18191_b200 import binding
    name, args = CALLS[fn]
    args = {k: Fake(*v) if isinstance(v, tuple) else Fake(v) if isinstance(v, torch.dtype) else v for k, v in args.items()}
    k = torch.zeros(4, 2, 16, 64, dtype=BF16)
    if "pages" in args:
        args["pages"] = tsfm.kv_pages(k, k, torch.zeros(2, 4, dtype=I32))
        args["pages"].device = 0
    args.update(change)
    reached = []

    class Library:
        def __getattr__(self, attr):
            return getattr(tsfm.lib, attr) if attr != name else lambda *a: reached.append(a) or 0
    monkeypatch.setattr(binding, "lib", Library())
    binding._torch_names()
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    try:
        getattr(binding, name)(*args.values())
    except tsfm.TsfmError as e:
        assert not reached
        return e.code
    assert len(reached) == 1
    return 0


@pytest.mark.parametrize("fn,name,kind", TENSORS)
def test_tensors_that_would_be_read_as_something_else(monkeypatch, fn, name, kind):
    right = kind[0] if isinstance(kind, tuple) else kind
    assert through_the_binding(monkeypatch, fn) == 0
    for wrong in (torch.int64, torch.float16, torch.float64, I32, F32, BF16):
        if wrong != right and name != "work":
            assert through_the_binding(monkeypatch, fn, **{name: Fake(wrong)}) == ARG, wrong
    assert through_the_binding(monkeypatch, fn, **{name: Fake(right, device=-1)}) == ARG       # host
    assert through_the_binding(monkeypatch, fn, **{name: Fake(right, device=1)}) == ARG        # another device
    assert through_the_binding(monkeypatch, fn, **{name: Fake(right, contiguous=False)}) == (ARG if isinstance(kind, tuple) else 0)
    import numpy as np
    assert through_the_binding(monkeypatch, fn, **{name: np.zeros(8, np.int32)}) == ARG
    assert through_the_binding(monkeypatch, fn, **{name: torch.zeros(8, dtype=right)}) == ARG


@pytest.mark.parametrize("fn", ["append", "attend", "evict"])
def test_pools_of_the_host_of_another_device_or_of_fewer_series(monkeypatch, fn):
    k = torch.zeros(4, 2, 16, 64, dtype=BF16)
    for rows, device, code in ((2, -1, ARG), (2, 1, ARG), (0, 0, ARG), (1, 0, ARG), (2, 0, 0), (3, 0, 0)):
        pool = tsfm.kv_pages(k, k, torch.zeros(rows, 4, dtype=I32))
        assert pool.device == -1
        pool.device = device
        assert through_the_binding(monkeypatch, fn, pages=pool) == code
    assert through_the_binding(monkeypatch, fn, pages=pages()) == 0                            # described by hand: the caller's own word
    # on another device than the current one, all of them
    from paper_2511_18191_b200 import binding
    binding._torch_names()
    name, args = CALLS[fn]
    args = {k: Fake(*v, device=1) if isinstance(v, tuple) else Fake(v, device=1) if isinstance(v, torch.dtype) else v for k, v in args.items()}
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    with pytest.raises(tsfm.TsfmError):
        getattr(tsfm, name)(*dict(args, pages=pages()).values())
