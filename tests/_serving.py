"""Plain 64-bit forms of the serving operators, and small caches to hold against them (not collected by pytest).

Tolerances of weights and outputs.  A logit is a sum of d_head products in 32 bits, off by at most (d_head + 3) 2^-24
times the sum of the products' magnitudes; with q of deviation 2 and d_head 128 that sum is about 163 / sqrt(128) 1.44 =
21 in the base-2 exponent, so a weight is off by at most 131 x 6e-8 x 21 x ln 2 = 1.2e-4 of itself (RTOL, with the
exponential's own 2^-22).  The errors are of random sign: over a whole output they leave about 1 / sqrt(d_head) of that,
1e-5; NORM allows twice that."""
from __future__ import annotations

import gc
import math

import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc

RTOL = 1.5e-4
NORM = 2e-5
TDT = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def collected():
    """Caches that a refusal's traceback still holds are freed with their module, not during a later test."""
    yield
    gc.collect()


def rotate(q, pos, rot, base=10000.0):
    """q [..., d] in 64 bits with its first `rot` columns rotated by halves at pos."""
    q = q.double()
    if rot == 0:
        return q
    i = torch.arange(rot // 2, dtype=torch.float64, device=q.device)
    a = float(pos) * base ** (-2.0 * i / rot)
    lo, hi = q[..., :rot // 2], q[..., rot // 2:rot]
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin(), q[..., rot:]], -1)


def attend(q, k, v, rows, scale):
    """(out [H, d], weights [H, rows]) of one query [H, d] over the given rows of k, v [H, n, d]."""
    z = torch.einsum("hd,hnd->hn", q, k[:, rows].double()) * scale
    w = torch.softmax(z, -1)
    return torch.einsum("hn,hnd->hd", w, v[:, rows].double()), w


def close(got, ref, what=""):
    got, ref = got.double().cpu(), ref.double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    norm = float((got - ref).norm() / ref.norm().clamp(min=1e-30))
    assert norm <= NORM, f"{what}: off by {norm:.3g} of the norm"


def close_weights(got, ref, what=""):
    got, ref = got.double().cpu(), ref.double().cpu()
    close(got, ref, what)
    worst = float(((got - ref).abs() - RTOL * ref.abs()).max())
    assert worst <= 1e-9, f"{what}: a weight is off by {worst:.3g} more than {RTOL} of itself"


def make(M, H, d, lens, dtype="f16", rot=0, spare=0, kinds=None, policy=kvc.POLICY_PAPER, seed=0, pos=None):
    """A cache whose sequences hold `lens` tokens of random K, V; (cache, per-sequence stored K [M][H, n, d], V)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    cap = [max(1, n) + spare for n in lens]
    cache = kvc.KVCache(M, H, d, cap, dtype, rotary_dim=rot, policy=policy)
    N = sum(lens)
    k, v = (torch.empty(M, N, H, d, dtype=TDT[dtype], device="cuda").normal_(generator=g) for _ in range(2))
    kinds = np.zeros(N, np.uint8) if kinds is None else np.concatenate(kinds)
    cache.append(k, v, lens, kinds, pos=pos)
    return cache, g


def rows_of(cache, s, n):
    """Stored K and V rows [M, H, n, d] of a sequence."""
    out = []
    for plane in (cache.k, cache.v):
        p = plane.view(cache.M, cache.H * cache.C, cache.d)
        base = cache.H * int(cache.offsets[s])
        cap = int(cache.capacity[s])
        out.append(p[:, base:base + cache.H * cap].view(cache.M, cache.H, cap, cache.d)[:, :, :n])
    return out


def per_row(cache, x, s, n):
    """A tensor in the rows' layout (scores, kept) as [M, H, n] of a sequence."""
    base, cap = cache.H * int(cache.offsets[s]), int(cache.capacity[s])
    return x.view(cache.M, cache.H * cache.C)[:, base:base + cache.H * cap].view(cache.M, cache.H, cap)[:, :, :n]


def query(cache, g, n_layers=None, sd=2.0):
    n = cache.M if n_layers is None else n_layers
    return torch.empty(n, cache.b, cache.H, cache.d, dtype=cache.torch_dtype, device="cuda").normal_(0.0, sd, generator=g)


def evict_reference(scores, keep, recent):
    """Earlier row numbers of the rows left of one stream, from its scores (float array of n rows)."""
    n = len(scores)
    a, cand = keep - recent, n - recent
    low = [-math.inf if x != x else x for x in scores]
    nan = [x != x for x in scores]
    order = sorted(range(cand), key=lambda i: (nan[i], -low[i], i))
    stay = set(order[:a])
    spare = iter(sorted(i for i in stay if i >= a))
    return [i if i in stay else next(spare) for i in range(a)] + list(range(cand, n))
