"""How far fp32 plans' products (three bf16 planes of each operand, six products for one) may be off over all results together, and what a plane less would
make of them.

u = 2^-24.  A sum of n products of random signs is about n^(1/2) of one; each of its additions is off by u / 3^(1/2) of the sum so far in the mean square at most, all of
them by u (n / 6)^(1/2) of the result, in any order; its own rounding, the sum of the small products and what the planes leave out (u of a product, see test_planes_ref.py)
are 4 u more.
"""
import math

import torch

U = 2.0 ** -24
TWO = 3.2e-6     # by how much products of random signs are off with two planes of each operand, at least (test_planes_ref.py)


def product_off(n):
    """Root mean square of a sum of n products' error, relative to that of the sums."""
    return (4 + math.sqrt(n / 6)) * U


def planes(v, count=3):
    """The first `count` bf16 planes of fp32 values, each what is left rounded to nearest (cut where that would be an infinity)."""
    left, out = v.float(), []
    for _ in range(count):
        p = left.bfloat16().float()
        cut = (left.view(torch.int32) & -65536).view(torch.float32)
        p = torch.where(torch.isinf(p), cut, p)
        out.append(p)
        left = left - p
    return out


def off(got, want):
    return float((got.double() - want).norm() / want.norm())
