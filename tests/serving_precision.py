"""How far the bf16 attention over pages may be off, and cases in which one rounding more shows.

Derivation, relative to sum p |v| unless said otherwise, u = 2^-24 (half a step of fp32):
  a score      products of bf16 are exact; a step of the tensor core adds 16 of them and the sum so far, of which each may lose a whole step
               of the largest: 17 x 2u a step, D / 16 steps, one more addition of two sums, all of peak = max sum |q k| |scale|
  p            scale in base 2 (three roundings of at most peak), the difference from the maximum (of at most 2 peak), the exponential
               (2^-22), in natural units: (8 + 8 peak) u
  sum of p     n additions in some order, and a rescaling (an exponential and a product) for a tile or a merge: (n + 64) u
  p v          p as two bf16 parts: the second is off by 2^-8 of a rest that is at most 2^-8 of p: 2^-16; then both parts' products, 17 x 2u for
               each 16 slots begun
  out          one rounding to bf16, 2^-8 of itself
"""
import math

import torch

from tests import serving_ref as ref

U32, UB = 2.0 ** -24, 2.0 ** -8


def score_error(D, peak):
    return (17 * D // 16 + 2) * 2 * U32 * peak + (8 + 8 * peak) * U32


def out_tolerance(D, n, o, absv, peak):
    rel = 2 * score_error(D, peak) + (n + 64) * U32 + 2.0 ** -16 + 2 * 17 * (n // 16 + 2) * 2 * U32
    return UB * o.abs() + rel[:, None] * absv


def lse_tolerance(D, n, z, peak):
    """A probability's error, the sum's, the logarithm and its products (of at most |z| + peak + log n)."""
    return score_error(D, peak) + (n + 64) * U32 + 4 * U32 * (z.abs() + peak + math.log(max(n, 1)) + 1)


def weight_tolerance(D, n, z, peak):
    """Relative, of one probability: its score's error, the log-sum's, the exponential of the difference."""
    return score_error(D, peak) + lse_tolerance(D, n, z, peak) + (8 + 4 * peak) * U32


def inputs(D, Hq, Hkv, M, lengths, seed):
    """q [B, M, Hq, D], k and v of each series [n, Hkv, D], bf16 on the host.  Values come in pairs of opposite sign beside a little noise, and two
    thirds of the slots have close scores: sums that all but cancel, so that what is lost in p is not hidden by the result's own rounding."""
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(len(lengths), M, Hq, D, generator=g).bfloat16()
    ks, vs = [], []
    for n in lengths:
        k = torch.randn(n, Hkv, D, generator=g) * 0.3
        v = torch.randn(n, Hkv, D, generator=g)
        v[1::2] = -v[0:n - n % 2:2] * (1 + 0.02 * torch.randn(v[1::2].shape, generator=g))
        ks.append(k.bfloat16())
        vs.append(v.bfloat16())
    return q, ks, vs


CASES = [(64, 1, 1, 1, [2, 8, 31, 64]), (128, 8, 1, 1, [3, 40, 130]), (32, 8, 2, 1, [6, 66]), (64, 5, 1, 3, [5, 64, 190]), (32, 3, 1, 4, [4, 63]),
         (128, 4, 1, 4, [7, 70]), (64, 8, 1, 5, [2, 9, 33, 129]), (32, 20, 1, 2, [12, 100]), (128, 9, 1, 9, [10, 65])]


def exact(q, k, v, n, M, m, scale):
    """Token m of M that are the last ones of n slots."""
    D = q.shape[-1]
    end = n - M + m + 1
    return (*ref.attention(q.double(), k.double(), v.double(), scale, 0, end), end, D)
