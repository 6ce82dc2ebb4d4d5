"""How near the decode over a cache of 4 bits comes on rows of the usual kind (not collected by pytest).

With q and k of deviation 1 and scale 1 / sqrt(d), in the base-2 exponent of a weight:
  a group's step (sum q (c - 8) + 8 sum q) and lo sum q are some 2.2 x 1.44 sqrt(32 / d) each; three roundings of them to 32 bits
  for each of d / 32 groups leave sqrt(3) x 2.2 x 1.44 x 2^-25 = 1.6e-7 (root mean square),
  the products' sums in the matrix unit, some six of a size near 1 cut at 2^-23, 1.7e-7,
  the query as two 16-bit parts, 2^-23 of its largest column: 0.6e-7.
A weight's exponential is off by 2^-22 at most (1e-7 root mean square), a weight times a step, in two 16-bit parts, by 2^-23, and a
sum of a thousand of those loses about as much again as its two halves, of lo + 8 step and of c - 8, are some five times what is
left of them: 5 x 2^-24 = 3e-7.  All of these are independent from row to row, as what they are multiplied by is, so an output is
off by their root mean square, 5e-7 of its norm.  USUAL is eight times that, for norms of a few dozen columns; it grows with the
logits where those are larger, and past a thousand rows with their root, as what is left of the two halves falls by it."""
from __future__ import annotations

import torch

from _packed import stored, values
from _serving import attend, rotate

USUAL = 4e-6


def expected(cache, s, q, n, scale, rows=None, pos=0):
    """out [M, H, d] of sequence s of n rows in 64 bits, over the given ones (all) of what the cache holds."""
    k, v = (values(*stored(cache, s, n, w)) for w in "kv")
    rows = range(n) if rows is None else rows
    return torch.stack([attend(rotate(q[m, s].cpu(), pos, cache.rotary_dim), k[m], v[m], rows, scale)[0] for m in range(cache.M)])


def close_usual(got, ref, what="", deviation=1.0):
    """deviation: what the bound grows by, of the logits or the root of thousands of rows."""
    got, ref = got.double().cpu(), ref.double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    off = float((got - ref).norm() / ref.norm().clamp(min=1e-300))
    assert off <= USUAL * max(1.0, deviation), f"{what}: off by {off:.3g} of the norm"


def close_groups(got, ref, what="", deviation=1.0):
    """Each group of 32 columns of [..., d] to its own size."""
    for a in range(0, got.shape[-1], 32):
        close_usual(got[..., a:a + 32], ref[..., a:a + 32], f"{what} columns {a}", deviation)
