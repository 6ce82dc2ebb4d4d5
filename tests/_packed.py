"""Plain forms of a cache of 4 bits (not collected by pytest).

Tolerance of the decode over it.  A logit is sum over the groups of step <q, c> + lo sum(q), so the magnitudes that are added
are |q| (|lo| + 15 step) a column instead of |q k|: a group of 32 standard normal values has lo near -2.1 and a range near 4.2,
so about 6.3 |q| against 0.8 |q| on average, eight times those of a decode over 16-bit rows, whose outputs are held to
NORM = 2e-5 (_serving.py).  The sum over the rows has the same ratio.  Hence NORM4 = 8 NORM.  The query goes into the products
as two 16-bit parts (2^-22 of the largest column, less than one of the roundings counted there), the weights times the steps
likewise."""
from __future__ import annotations

import numpy as np
import torch

import paper_2310_08152_gb300 as kvc
from _serving import NORM, TDT

NORM4 = 8 * NORM
N, CL, CR = kvc.NORMAL, kvc.CL, kvc.CR


def quantise(x):
    """(codes uint8 [..., d], step, lo [..., groups] in 64 bits) of rows of a 16-bit type, by their definition."""
    dt, d = x.dtype, x.shape[-1]
    bits, least = (11, -24) if dt == torch.float16 else (8, -133)
    x = x.cpu().double()
    codes, steps, los = torch.zeros(x.shape, dtype=torch.uint8), [], []
    for a in range(0, d, 32):
        part = x[..., a:a + 32]
        lo = part.amin(-1)
        s = (part.amax(-1) - lo).float().numpy() / np.float32(15)
        s = np.where(s < np.float32(2.0 ** -126), np.float32(0), s).astype(np.float64)
        unit = np.exp2(np.maximum(np.frexp(s)[1] - bits, least).astype(np.float64))
        step = torch.from_numpy(np.ceil(s / unit) * unit)
        inv = np.divide(np.float32(1), step.numpy().astype(np.float32), out=np.zeros(step.shape, np.float32), where=step.numpy() > 0)
        t = (part - lo[..., None]).float().numpy() * inv[..., None]
        codes[..., a:a + 32] = torch.from_numpy(np.rint(t).clip(0, 15).astype(np.uint8))
        steps.append(step)
        los.append(lo)
    return codes, torch.stack(steps, -1), torch.stack(los, -1)


def values(codes, step, lo):
    """What the codes stand for, in 64 bits."""
    x = torch.empty(codes.shape, dtype=torch.float64)
    for g, a in enumerate(range(0, codes.shape[-1], 32)):
        x[..., a:a + 32] = lo[..., g:g + 1].double() + step[..., g:g + 1].double() * codes[..., a:a + 32].double()
    return x


def held(x):
    return values(*quantise(x)).to(x.device)


def stored(cache, s, n, which="k"):
    """(codes [M, H, n, d], step, lo [M, H, n, groups]) that a cache of 4 bits holds for rows [0, n) of sequence s."""
    M, H, d, G = cache.M, cache.H, cache.d, (cache.d + 31) // 32
    raw = getattr(cache, which).cpu()
    rows = M * H * cache.C
    code = raw[:rows * d // 2].view(rows, d // 2)
    start = (rows * d // 2 + 255) // 256 * 256
    pair = raw[start:start + rows * G * 4].view(cache.torch_dtype).view(rows, G, 2)
    cap = (int(cache.capacity[s]) + 3) // 4 * 4
    at = torch.tensor([[[m * H * cache.C + H * int(cache.offsets[s]) + h * cap + i for i in range(n)] for h in range(H)] for m in range(M)],
                      dtype=torch.long).view(M, H, n)
    c, p = code[at], pair[at]
    return torch.stack([c & 15, c >> 4], -1).flatten(-2), p[..., 1].double(), p[..., 0].double()


def fill(M, H, d, lens, dtype="f16", rot=0, spare=0, kinds=None, policy=kvc.POLICY_PAPER, seed=0, bits=4, pos=None):
    """A cache of the given rows' bits that holds `lens` random tokens; (cache, generator, K [M, N, H, d], V)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    cache = kvc.KVCache(M, H, d, [max(1, n) + spare for n in lens], dtype, rotary_dim=rot, policy=policy, bits=bits)
    n_tok = sum(lens)
    k, v = (torch.empty(M, n_tok, H, d, dtype=TDT[dtype], device="cuda").normal_(generator=g) for _ in range(2))
    kinds = np.zeros(n_tok, np.uint8) if kinds is None else np.concatenate(kinds)
    if n_tok:
        cache.append(k, v, lens, kinds, pos=pos)
    return cache, g, k, v


def unpack16(cache):
    """A 16-bit copy of a cache of 4 bits."""
    wide = kvc.KVCache(cache.M, cache.H, cache.d, cache.capacity, cache.dtype, rotary_dim=cache.rotary_dim, policy=cache.policy)
    wide.copy_from(cache, range(cache.b), range(cache.b))
    return wide


def tokens(x, lens, s):
    """Rows [M, H, n, d] of sequence s of tokens [M, N, H, d]."""
    a = sum(lens[:s])
    return x[:, a:a + lens[s]].transpose(1, 2)


def close4(got, ref, what=""):
    got, ref = got.double().cpu(), ref.double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    norm = float((got - ref).norm() / ref.norm().clamp(min=1e-30))
    assert norm <= NORM4, f"{what}: off by {norm:.3g} of the norm"
