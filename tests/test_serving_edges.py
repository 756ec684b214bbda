"""Serving over a cache of pages, at the edges of what a call may be given: what needs no GPU."""
import os
import shutil
import subprocess

import pytest

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
