"""Random histories over a cache of 16 bits and one of 4: appends, spans freed, cuts, copies within and between the caches and
freed sequences, against a plain record of every sequence's tokens."""
import math

import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc
from _packed import CL, CR, N, close4, held, quantise, stored
from _serving import collected, rows_of  # noqa: F401

pytestmark = pytest.mark.gpu


class Sequence:
    """Tokens' kinds and the stored ones' history indices, and each token's K and V rows as the cache holds them ([M, H, d],
    16 bits; of a 4-bit cache the rows that were quantised)."""

    def __init__(self):
        self.kinds, self.rows, self.k, self.v, self.freed = [], [], [], [], []

    def copy(self):
        c = Sequence()
        c.kinds, c.rows, c.k, c.v, c.freed = list(self.kinds), list(self.rows), list(self.k), list(self.v), list(self.freed)
        return c

    def spans(self):
        out, cl = [], -1
        for j, k in enumerate(self.kinds):
            if k == CL:
                cl = j
            elif k == CR:
                out.append((cl, j))
                cl = -1
        return out, cl

    def pending(self):
        return [s for s in self.spans()[0] if s not in self.freed]

    def seen(self):
        """Stored rows that the last token sees (numbers among the stored ones), or None where that is refused."""
        t = len(self.kinds) - 1
        if self.kinds[t] == CL:
            return [len(self.rows) - 1]
        hidden, runs = set(), 0
        closed, cl = self.spans()
        for a, z in closed:
            if (a, z) in self.freed:
                continue
            hidden |= set(range(a, z)) if z < t else {a}
        if cl >= 0:
            hidden.add(cl)
        vis = [j not in hidden for j in self.rows]
        runs = sum(1 for i, x in enumerate(vis) if not x and (i == 0 or vis[i - 1]))
        return None if runs > 1 else [i for i, x in enumerate(vis) if x]


def check(cache, seqs, g):
    lens = [len(s.rows) for s in seqs]
    assert cache.lengths()[0].tolist() == lens
    for i, s in enumerate(seqs):
        if s.rows:
            lay = cache.masked_reference_layout(i)
            assert lay["stored_orig"].tolist() == s.rows and lay["kinds"].tolist() == s.kinds
            assert cache.pending_spans(i) == s.pending()
    views = [s.seen() if s.kinds else [] for s in seqs]
    for i, s in enumerate(seqs):
        if not s.rows:
            continue
        for w in "kv":
            x = torch.stack([getattr(s, w)[j] for j in s.rows], 2)  # [M, H, n, d]
            if cache.bits == 4:
                for a, b in zip(stored(cache, i, lens[i], w), quantise(x)):
                    assert torch.equal(a, b), (i, w)
            else:
                assert torch.equal(rows_of(cache, i, lens[i])["kv".index(w)], x), (i, w)
    if any(v is None for v in views) or not any(lens):
        return
    q = torch.empty(cache.M, cache.b, cache.H, cache.d, dtype=cache.torch_dtype, device="cuda").normal_(0, 2, generator=g)
    out = cache.decode_attention_layers(q, 1 / math.sqrt(cache.d))
    for i, (s, v) in enumerate(zip(seqs, views)):
        if not s.rows:
            continue
        k, x = (torch.stack([getattr(s, w)[s.rows[j]] for j in v], 2) for w in "kv")
        if cache.bits == 4:
            k, x = held(k), held(x)
        p = torch.softmax(torch.einsum("mhd,mhnd->mhn", q[:, i].double(), k.double()) / math.sqrt(cache.d), -1)
        close4(out[:, i], torch.einsum("mhn,mhnd->mhd", p, x.double()), f"sequence {i}")


@pytest.mark.parametrize("d,dtype,seed", [(64, "f16", 0), (80, "bf16", 1), (96, "f16", 2), (128, "bf16", 3), (80, "f16", 4)])
def test_random_histories(d, dtype, seed):
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    M, H, b, cap = 2, 2, 5, 211
    caches = [kvc.KVCache(M, H, d, [cap] * b, dtype, bits=bits) for bits in (16, 4)]
    books = [[Sequence() for _ in range(b)] for _ in caches]
    for step in range(60):
        c = int(rng.integers(0, 2))
        cache, seqs = caches[c], books[c]
        act = rng.choice(["append", "append", "append", "free", "cut", "copy", "other", "drop"])
        if act == "append":
            n_new = [int(rng.integers(0, 1 + min(int(rng.choice([1, 3, 40])), cap - len(s.rows)))) for s in seqs]
            kinds, new = [], []
            for s, n in zip(seqs, n_new):
                open_ = s.spans()[1] >= 0
                part = []
                for _ in range(n):
                    k = N
                    if not open_ and rng.random() < 0.1:
                        k, open_ = CL, True
                    elif open_ and rng.random() < 0.2:
                        k, open_ = CR, False
                    part.append(k)
                kinds += part
                new.append(part)
            if not kinds:
                continue
            k, v = (torch.empty(M, len(kinds), H, d, dtype=cache.torch_dtype, device="cuda").normal_(generator=g) for _ in range(2))
            if rng.random() < 0.5:
                cache.append(k, v, n_new, np.array(kinds, np.uint8))
            else:
                for m in range(M):
                    cache.append(k[m].contiguous(), v[m].contiguous(), n_new, np.array(kinds, np.uint8), layer=m)
            t = 0
            for s, part in zip(seqs, new):
                s.rows += range(len(s.kinds), len(s.kinds) + len(part))
                s.kinds += part
                s.k += [k[:, t + i] for i in range(len(part))]
                s.v += [v[:, t + i] for i in range(len(part))]
                t += len(part)
        elif act == "free":
            spans = [(i, a, z) for i, s in enumerate(seqs) for a, z in s.pending() if rng.random() < 0.8]
            if spans:
                cache.compress_spans(*zip(*spans))
                for i, a, z in spans:
                    seqs[i].freed.append((a, z))
                    seqs[i].rows = [j for j in seqs[i].rows if not a <= j < z]
        elif act == "cut":
            to = [-1] * b
            for i, s in enumerate(seqs):
                if s.kinds and rng.random() < 0.6:
                    n = int(rng.integers(max(1, len(s.kinds) - 9), len(s.kinds) + 1))
                    if not any(a < n <= z for a, z in s.freed):
                        to[i] = n
            cache.truncate(to)
            for s, n in zip(seqs, to):
                if n >= 0:
                    s.kinds, s.k, s.v = s.kinds[:n], s.k[:n], s.v[:n]
                    s.rows = [j for j in s.rows if j < n]
                    s.freed = [(a, z) for a, z in s.freed if z < n]
        elif act == "drop":
            i = int(rng.integers(0, b))
            cache.truncate([0 if j == i else -1 for j in range(b)])
            seqs[i] = Sequence()
        elif act == "copy":
            order = rng.permutation(b).tolist()
            n = int(rng.integers(1, b))
            dst, src = order[:n], [order[n + int(rng.integers(0, b - n))] for _ in range(n)]
            cache.copy_from(cache, dst, src)
            for a, z in zip(dst, src):
                seqs[a] = seqs[z].copy()
        else:  # from the other cache
            other = books[1 - c]
            n = int(rng.integers(1, b + 1))
            dst = rng.permutation(b)[:n].tolist()
            src = [int(x) for x in rng.integers(0, b, n)]
            cache.copy_from(caches[1 - c], dst, src)
            for a, z in zip(dst, src):
                seqs[a] = other[z].copy()
                if c == 0:  # from 4 bits: the values that those stand for
                    seqs[a].k = [held(x).float().to(x.dtype) for x in seqs[a].k]
                    seqs[a].v = [held(x).float().to(x.dtype) for x in seqs[a].v]
        check(cache, seqs, g)
    for cache in caches:
        assert cache.device_status() == 0
