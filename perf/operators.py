"""The cache's operators for many samples of one prompt under a bounded cache, as cases that can be timed and compared.

Four kinds of pass, each through the package's public calls:

  scored   the decode step's attention that also adds each row's attention weight to the row's score
  prompt   the attention weights of a prompt's last queries, added to the scores of one layer's rows
  evict    a block of tokens is appended and every (layer, sequence, head) stream is brought back to its budget: the
           recent rows and those with the largest scores stay.  The scores are written before each pass, in the place
           of the decode steps that would have moved them
  shared   the decode step's attention of samples that share their prompt's rows, held once in a cache of their own

Sizes are those of the repository's workloads (OPT-1.3B-, OPT-2.7B- and 3B-rotary-shaped caches, the paper's 8 samples of
a prompt and prefixes of 800 tokens), and generic ones.  K and V are standard normal in the cache type, q has twice their
deviation, so that the weights of a row spread over several orders of magnitude; all are made from the seed on the GPU.
A stored row of a rotary cache holds its rotated key, so K is what the cache holds in either case.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False  # set from outside: False computes the plain forms, True calls the package

DEVICE = "cuda:0"
NORMAL, CL, CR = 0, 1, 2
_TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}
_NEVER = 1 << 30
_ROPE_BASE = 10000.0

# Fields that a case may leave out.
_DEFAULTS = {"dtype": "f16", "rot": 0, "open": False, "interior": 0, "shape_seed": 0, "lmin": 0}


def listed():
    return [
        # The smallest call: one layer of one short sequence; latency is all there is.
        {"name": "scored_one_layer", "kind": "scored", "M": 1, "H": 8, "d": 64, "b": 1, "lmax": 257},
        # A serving step of an OPT-1.3B-shaped batch whose cache is kept at about a thousand rows a sequence.
        {"name": "scored_opt1.3b", "kind": "scored", "M": 24, "H": 32, "d": 64, "b": 16, "lmax": 1024},
        # Sequences of very different lengths, bf16, d_head 80, some inside an open span (its <CL> row is hidden).
        {"name": "scored_ragged_bf16", "kind": "scored", "M": 4, "H": 32, "d": 80, "dtype": "bf16", "b": 32, "lmin": 64, "lmax": 4096,
         "open": True, "shape_seed": 3},
        # A short prompt judged by its last tokens: latency.
        {"name": "prompt_short", "kind": "prompt", "H": 8, "d": 64, "b": 1, "lmax": 700, "nq": 32},
        # Long prompts of different lengths judged by an observation window, bf16.
        {"name": "prompt_window_bf16", "kind": "prompt", "H": 32, "d": 128, "dtype": "bf16", "b": 6, "lmin": 3000, "lmax": 8191, "nq": 64,
         "shape_seed": 1},
        # Whole prompts with their sentinel spans still stored, as in the paper's loop before the spans are freed.
        {"name": "prompt_opt1.3b", "kind": "prompt", "H": 32, "d": 64, "b": 4, "lmax": 2048, "nq": 2048, "interior": 32},
        # A token more than the budget in a small cache: latency.
        {"name": "evict_small_step", "kind": "evict", "M": 2, "H": 8, "d": 64, "b": 2, "keep": 500, "recent": 61, "blk": 1},
        # Every step of an OPT-1.3B-shaped batch brings each stream back to its budget.
        {"name": "evict_opt1.3b_step", "kind": "evict", "M": 24, "H": 32, "d": 64, "b": 16, "keep": 1024, "recent": 128, "blk": 1},
        # Blocks of 256 tokens between evictions, bf16, OPT-2.7B heads.
        {"name": "evict_blocks_bf16", "kind": "evict", "M": 8, "H": 32, "d": 80, "dtype": "bf16", "b": 8, "keep": 1536, "recent": 200,
         "blk": 256},
        # Eight samples of one short prompt, a layer: latency.
        {"name": "shared_one_layer", "kind": "shared", "M": 1, "H": 8, "d": 64, "P": 1, "G": 8, "lmax": 200, "lown": 5},
        # The paper's 8 samples of each prefix of 800 tokens, 3B rotary shape, all layers, up to 100 own tokens.
        {"name": "shared_8_samples", "kind": "shared", "M": 32, "H": 32, "d": 80, "rot": 80, "P": 8, "G": 8, "lmax": 800, "lown": 100,
         "shape_seed": 2},
        # Many samples of one long document, bf16, wide heads.
        {"name": "shared_long_bf16", "kind": "shared", "M": 2, "H": 32, "d": 128, "dtype": "bf16", "P": 1, "G": 64, "lmax": 32768,
         "lown": 300, "shape_seed": 4},
    ]


# ------------------------------------------------------------------------------------------
# Drawn cases
# ------------------------------------------------------------------------------------------

def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        c = _draw_once(rng)
        w = work(c)
        # no dearer than the largest listed case of its kind, and more than a few rows
        most = {"scored": (3.6e9, 1e30), "prompt": (1e9, 3.4e10), "evict": (4e9, 1e30), "shared": (3.4e9, 9e10)}[c["kind"]]
        if 2e4 < w["bytes"] <= most[0] and w["flops"] <= most[1] and _plain_bytes(c) < 1.2e10:
            return c


def _draw_once(rng):
    kind = rng.choice(["scored", "prompt", "evict", "shared"])
    d = rng.choice([64, 64, 80, 96, 128])
    c = {"kind": kind, "H": rng.choice([4, 8, 12, 16, 20, 32, 32, 40]), "d": d, "dtype": rng.choice(["f16", "bf16"]),
         "shape_seed": rng.randrange(1 << 20)}
    if kind == "scored":
        c.update(M=_log_int(rng, 1, 24), b=_log_int(rng, 1, 64), lmax=_log_int(rng, 64, 16384), open=rng.random() < 0.4, rot=rng.choice([0, 0, d]))
    elif kind == "prompt":
        c.update(b=_log_int(rng, 1, 16), lmax=_log_int(rng, 64, 16384), interior=rng.choice([0, 0, 19, 44]), rot=rng.choice([0, 0, d]))
        c["nq"] = _log_int(rng, 1, c["lmax"])
    elif kind == "evict":
        c.update(M=_log_int(rng, 1, 24), b=_log_int(rng, 1, 16), keep=_log_int(rng, 64, 4096), blk=_log_int(rng, 1, 512))
        c["recent"] = _log_int(rng, 1, max(2, c["keep"] // 2))
    else:
        c.update(M=_log_int(rng, 1, 32), P=_log_int(rng, 1, 16), G=_log_int(rng, 1, 128), lmax=_log_int(rng, 64, 32768),
                 lown=_log_int(rng, 1, 512), rot=rng.choice([0, 0, d]))
    if kind in ("scored", "prompt", "shared"):
        c["lmin"] = 0 if rng.random() < 0.4 else max(1, int(c["lmax"] * rng.uniform(0.05, 0.9)))
    return c


def _plain_bytes(c):
    """The largest temporary of the plain form."""
    if c["kind"] == "prompt":
        return 4 * c["b"] * c["H"] * min(c["nq"], c["lmax"]) * c["lmax"]
    if c["kind"] == "shared":
        return 4 * c["M"] * c["H"] * c["P"] * c["lmax"] * max(c["G"], c["d"])
    if c["kind"] == "scored":
        return 4 * c["M"] * c["H"] * c["b"] * c["lmax"] * c["d"]
    return 4 * c["M"] * c["H"] * c["b"] * (c["keep"] + c["blk"]) * c["d"]


# ------------------------------------------------------------------------------------------
# What a case looks like (plain numpy)
# ------------------------------------------------------------------------------------------

def _case(case):
    return dict(_DEFAULTS, **case)


def _lens(c, n):
    """n lengths in [lmin, lmax] (all lmax where lmin is 0), the first of them lmax."""
    if not c["lmin"]:
        return [c["lmax"]] * n
    rng = random.Random(c["shape_seed"])
    return [c["lmax"]] + [rng.randint(c["lmin"], c["lmax"]) for _ in range(n - 1)]


def _own_lens(c):
    rng = random.Random(c["shape_seed"] + 1)
    return [rng.randint(1, c["lown"]) for _ in range(c["P"] * c["G"])]


def _open_rows(c, lens):
    """The row of each sequence's open <CL>, or -1: every other sequence with rows enough has one, a few rows from its end."""
    rng = random.Random(c["shape_seed"] + 2)
    return [n - 1 - rng.randint(1, 20) if c["open"] and s % 2 == 0 and n > 30 else -1 for s, n in enumerate(lens)]


def _span_kinds(n, interior):
    """Spans of `interior` tokens, one in every 64-token block: <CL> at its eighth token."""
    k = np.zeros(n, np.uint8)
    if interior:
        for a in range(7, n - interior - 1, 64):
            k[a], k[a + interior + 1] = CL, CR
    return k


def _hid(kinds):
    """The last query that sees each row (the <CR> of a span around it; a <CL> itself alone)."""
    h = np.full(kinds.size, _NEVER, np.int64)
    cl = -1
    for j, k in enumerate(kinds):
        if k == CL:
            h[j], cl = j, j
        elif k == CR:
            h[cl + 1:j] = j
    return h


def _tied_positions(kinds):
    normal = kinds == NORMAL
    return np.maximum(np.cumsum(normal) - 1, 0).astype(np.int64)


def work(case):
    c = _case(case)
    H, d = c["H"], c["d"]
    row = 4 * d  # a K and a V row
    if c["kind"] == "scored":
        n = c["M"] * H * sum(_lens(c, c["b"]))
        return {"bytes": n * (row + 8) + c["M"] * c["b"] * H * 6 * d, "flops": 4 * d * n}
    if c["kind"] == "prompt":
        rows = queries = pairs = 0
        for n in _lens(c, c["b"]):
            q = min(c["nq"], n)
            kinds = _span_kinds(n, c["interior"])
            i = np.arange(n)
            first = np.maximum(i, n - q)  # the queries that see row i, a <CL> query aside
            last = np.minimum(_hid(kinds), n - 1)
            p = int(np.maximum(last - first + 1, 0).sum())
            vis = np.where(kinds == CL, 0, 1)
            # a <CL> query sees itself alone
            for t in np.nonzero(kinds == CL)[0]:
                if t >= n - q:
                    p -= int(((i <= t) & (_hid_cached(n, c["interior"]) >= t)).sum()) - 1
            del vis
            rows, queries, pairs = rows + n, queries + q, pairs + p
        return {"bytes": H * (rows * (2 * d + 8) + queries * 2 * d), "flops": 2 * d * H * pairs}
    if c["kind"] == "evict":
        # scores read; new rows read and written; about a (candidates dropped / candidates) share of the rows below the
        # boundary replaced; the recent rows moved; the kept rows' numbers and scores written
        cand, a = c["keep"] + c["blk"] - c["recent"], c["keep"] - c["recent"]
        moved = a * c["blk"] / cand + c["recent"]
        n = c["M"] * c["b"] * H
        return {"bytes": n * (4 * (c["keep"] + c["blk"]) + 2 * row * (moved + c["blk"]) + 8 * c["keep"]), "flops": 0}
    lens, lown = _lens(c, c["P"]), _own_lens(c)
    rows = sum(lens) + sum(lown)
    pairs = c["G"] * sum(lens) + sum(lown)
    n = c["M"] * H
    return {"bytes": n * (rows * row + c["P"] * c["G"] * 6 * d), "flops": 4 * d * n * pairs}


_HID = {}


def _hid_cached(n, interior):
    if (n, interior) not in _HID:
        _HID[n, interior] = _hid(_span_kinds(n, interior))
    return _HID[n, interior]


# ------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) & 0x7FFFFFFF)
    return g


def _normal(shape, dtype, g, sd=1.0):
    x = torch.empty(shape, dtype=_TORCH[dtype], device=DEVICE)
    return x.normal_(0.0, sd, generator=g)


def _rows(c, M, lens, g):
    """K and V [M, b, H, cap, d], zero past each length."""
    cap = max(lens)
    k, v = (_normal((M, len(lens), c["H"], cap, c["d"]), c["dtype"], g) for _ in range(2))
    for s, n in enumerate(lens):
        k[:, s, :, n:] = 0
        v[:, s, :, n:] = 0
    return k, v


def _inputs(c, seed):
    g = _gen(seed)
    H, d, kind = c["H"], c["d"], c["kind"]
    x = {}
    if kind == "scored":
        lens = _lens(c, c["b"])
        x["k"], x["v"] = _rows(c, c["M"], lens, g)
        x["q"] = _normal((c["M"], c["b"], H, d), c["dtype"], g, 2.0)
    elif kind == "prompt":
        lens = _lens(c, c["b"])
        x["k"], _ = _rows(c, 1, lens, g)
        x["q"] = _normal((sum(min(c["nq"], n) for n in lens), H, d), c["dtype"], g, 2.0)
    elif kind == "evict":
        n = c["keep"] + c["blk"]
        x["k"], x["v"] = _rows(c, c["M"], [n] * c["b"], g)
        x["k_new"], x["v_new"] = (_normal((c["M"], c["b"] * c["blk"], H, d), c["dtype"], g) for _ in range(2))
        # sums of attention weights: a few large ones, many small, some equal
        w = torch.empty(c["M"], c["b"], H, n, device=DEVICE).normal_(0.0, 2.0, generator=g).exp_()
        x["fresh"] = w.bfloat16().float()
    else:
        lens, lown = _lens(c, c["P"]), _own_lens(c)
        x["k"], x["v"] = _rows(c, c["M"], lens, g)
        x["ko"], x["vo"] = _rows(c, c["M"], lown, g)
        x["q"] = _normal((c["M"], c["P"] * c["G"], H, d), c["dtype"], g, 2.0)
    return x


def _cache(c, M, lens, k, v, kinds=None, pos=None):
    """A cache of the package that holds the rows k, v [M, b, H, cap, d]."""
    import paper_2310_08152_gb300 as kvc

    b, cap = len(lens), k.shape[3]
    cache = kvc.KVCache(M, c["H"], c["d"], [cap] * b, c["dtype"], rotary_dim=c["rot"], rope_base=_ROPE_BASE)
    N = sum(lens)
    kinds = np.zeros(N, np.uint8) if kinds is None else kinds
    blank = torch.zeros(N, c["H"], c["d"], dtype=k.dtype, device=DEVICE)
    for m in range(M):
        cache.append(blank, blank, lens, kinds, pos=pos, layer=m)
    cache.k.view(k.shape).copy_(k)
    cache.v.view(k.shape).copy_(k if v is None else v)
    return cache


def prepare(case, seed):
    c = _case(case)
    x = _inputs(c, seed)
    s = {"case": c, **x, "scale": 1.0 / math.sqrt(c["d"])}
    dev = lambda a: torch.tensor(np.asarray(a), device=DEVICE)  # noqa: E731
    if c["kind"] == "scored":
        lens = _lens(c, c["b"])
        hidden = _open_rows(c, lens)
        s["lens"], s["hidden"], s["pos"] = dev(lens), dev(hidden), dev([n - 1 - (h >= 0) for n, h in zip(lens, hidden)])
        s["scores"] = torch.zeros(c["M"], c["b"], c["H"], max(lens), device=DEVICE)
        if own:
            kinds = np.concatenate([np.where(np.arange(n) == h, CL, NORMAL) for n, h in zip(lens, hidden)]).astype(np.uint8)
            s["cache"] = _cache(c, c["M"], lens, x["k"], x["v"], kinds)
            s["cache"].attach_scores(s["scores"])
    elif c["kind"] == "prompt":
        lens = _lens(c, c["b"])
        nq, cap = [min(c["nq"], n) for n in lens], max(lens)
        kinds = [_span_kinds(n, c["interior"]) for n in lens]
        mq = max(nq)
        hid, cl, at, pos = (np.zeros((c["b"], w), np.int64) for w in (cap, mq, mq, mq))
        tok = np.zeros((c["b"], mq), np.int64)
        t = 0
        for i, (n, m, k) in enumerate(zip(lens, nq, kinds)):
            hid[i, :n] = _hid(k)
            hid[i, n:] = -1
            cl[i, :m], pos[i, :m] = k[n - m:] == CL, _tied_positions(k)[n - m:]
            at[i] = -1  # no query
            at[i, :m] = np.arange(n - m, n)
            tok[i, :m] = np.arange(t, t + m)
            t += m
        s.update(hid=dev(hid), is_cl=dev(cl.astype(bool)), at=dev(at), pos=dev(pos), tok=dev(tok), nq=nq)
        s["scores"] = torch.zeros(1, c["b"], c["H"], cap, device=DEVICE)
        if own:
            s["cache"] = _cache(c, 1, lens, x["k"], None, np.concatenate(kinds))
            s["cache"].attach_scores(s["scores"])
    elif c["kind"] == "evict":
        s["scores"] = torch.zeros_like(x["fresh"])
        s["kept"] = torch.zeros(x["fresh"].shape, dtype=torch.int32, device=DEVICE)
        if own:
            lens = [c["keep"]] * c["b"]
            s["cache"] = _cache(c, c["M"], lens, x["k"], x["v"])
            s["cache"].attach_scores(s["scores"])
            s["n_new"], s["kinds"] = np.full(c["b"], c["blk"], np.int32), np.zeros(c["b"] * c["blk"], np.uint8)
    else:
        lens, lown = _lens(c, c["P"]), _own_lens(c)
        parent = np.repeat(np.arange(c["P"], dtype=np.int32), c["G"])
        s["lens"], s["lown"] = dev(lens), dev(lown)
        s["pos"] = dev([lens[p] + n - 1 for p, n in zip(parent, lown)])
        if own:
            pos = np.concatenate([lens[p] + np.arange(n) for p, n in zip(parent, lown)]).astype(np.int32)
            s["prefix"] = _cache(c, c["M"], lens, x["k"], x["v"])
            s["cache"] = _cache(c, c["M"], lown, x["ko"], x["vo"], pos=pos)
            s["cache"].set_prefix(s["prefix"], parent)
            s["out"] = torch.zeros(x["q"].shape, dtype=torch.float32, device=DEVICE)
    if c["kind"] == "scored":
        s["out"] = torch.zeros(x["q"].shape, dtype=torch.float32, device=DEVICE)
    return s


# ------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        cache = state["cache"]
        if c["kind"] == "scored":
            cache.decode_attention_scored(state["q"], state["scale"], out=state["out"])
            return {"out": state["out"], "scores": state["scores"]}
        if c["kind"] == "prompt":
            cache.score_prompt(0, state["q"], state["nq"], state["scale"])
            return {"scores": state["scores"]}
        if c["kind"] == "evict":
            cache.append(state["k_new"], state["v_new"], state["n_new"], state["kinds"])
            state["scores"].copy_(state["fresh"])
            cache.evict(c["keep"], c["recent"], kept=state["kept"])
            shape, keep = state["k"].shape, c["keep"]
            return {"k": cache.k.view(shape)[..., :keep, :], "v": cache.v.view(shape)[..., :keep, :], "scores": state["scores"],
                    "kept": state["kept"][..., :keep]}
        cache.decode_attention_shared(state["q"], state["scale"], out=state["out"])
        return {"out": state["out"]}
    return {"scored": _plain_scored, "prompt": _plain_prompt, "evict": _plain_evict, "shared": _plain_shared}[c["kind"]](state)


def _rotated(q, pos, rot):
    """q [..., d] in 32 bits, its first `rot` columns rotated by halves at `pos` (of q's shape without its last axis, or
    broadcast to it); the angles are reduced in 64 bits."""
    q = q.float()
    if not rot:
        return q
    i = torch.arange(rot // 2, device=q.device, dtype=torch.float64)
    a = pos.double()[..., None] * _ROPE_BASE ** (-2.0 * i / rot)
    cs, sn = a.cos().float(), a.sin().float()
    lo, hi = q[..., :rot // 2], q[..., rot // 2:rot]
    return torch.cat([lo * cs - hi * sn, hi * cs + lo * sn, q[..., rot:]], -1)


def _plain_scored(s):
    c = s["case"]
    q = _rotated(s["q"], s["pos"][None, :, None], c["rot"])
    z = (s["k"].float() @ q[..., None])[..., 0] * s["scale"]  # [M, b, H, cap]
    i = torch.arange(z.shape[-1], device=z.device)
    seen = (i < s["lens"][:, None]) & (i != s["hidden"][:, None])
    z = z.masked_fill(~seen[None, :, None], -math.inf)
    p = (z - z.amax(-1, keepdim=True)).exp()
    w = p / p.sum(-1, keepdim=True)
    out = (w[..., None, :] @ s["v"].float())[..., 0, :]
    s["scores"] += w
    return {"out": out, "scores": s["scores"]}


def _plain_prompt(s):
    c = s["case"]
    q = _rotated(s["q"][s["tok"]], s["pos"][..., None], c["rot"]).transpose(1, 2)  # [b, H, mq, d]
    z = (q @ s["k"][0].float().transpose(-1, -2)) * s["scale"]
    i, at = torch.arange(z.shape[-1], device=z.device), s["at"][..., None]
    seen = (i <= at) & (at <= s["hid"][:, None, :]) & (~s["is_cl"][..., None] | (i == at))
    z = z.masked_fill(~seen[:, None], -math.inf)
    m = z.amax(-1, keepdim=True).clamp(min=-1e30)
    p = (z - m).exp()
    w = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    s["scores"][0] += w.sum(-2)
    return {"scores": s["scores"]}


def _plain_evict(s):
    c = s["case"]
    keep, recent, blk = c["keep"], c["recent"], c["blk"]
    a, n = keep - recent, keep + blk
    for cache, new in ((s["k"], s["k_new"]), (s["v"], s["v_new"])):
        cache[..., keep:, :] = new.view(c["M"], c["b"], blk, c["H"], c["d"]).transpose(2, 3)
    s["scores"].copy_(s["fresh"])
    cand = s["scores"][..., :n - recent]
    best = torch.sort(cand, dim=-1, descending=True, stable=True).indices[..., :a]
    stays = torch.zeros(cand.shape, dtype=torch.bool, device=cand.device).scatter_(-1, best, True)
    # the j-th row below the new boundary that goes is replaced by the j-th row beyond it that stays
    hole = ~stays[..., :a]
    beyond = torch.sort(stays[..., a:].byte(), dim=-1, descending=True, stable=True).indices + a
    which = (hole.cumsum(-1) - 1).clamp(min=0, max=beyond.shape[-1] - 1)
    i = torch.arange(a, device=cand.device).expand(hole.shape)
    src = torch.where(hole, beyond.gather(-1, which), i)
    tail = torch.arange(n - recent, n, device=cand.device).expand(*src.shape[:-1], recent)
    src = torch.cat([src, tail], -1)
    s["kept"][..., :keep] = src
    s["scores"][..., :keep] = s["scores"].gather(-1, src)
    s["scores"][..., keep:] = 0
    at = src[..., None].expand(*src.shape, c["d"])
    for cache in (s["k"], s["v"]):
        cache[..., :keep, :] = cache.gather(-2, at)
    return {"k": s["k"][..., :keep, :], "v": s["v"][..., :keep, :], "scores": s["scores"], "kept": s["kept"][..., :keep]}


def _plain_shared(s):
    c = s["case"]
    M, P, G, H, d = c["M"], c["P"], c["G"], c["H"], c["d"]
    q = _rotated(s["q"], s["pos"][None, :, None], c["rot"])
    zo = (s["ko"].float() @ q[..., None])[..., 0] * s["scale"]  # [M, b, H, own rows]
    zo = zo.masked_fill(torch.arange(zo.shape[-1], device=zo.device) >= s["lown"][:, None, None], -math.inf)
    qg = q.view(M, P, G, H, d).transpose(2, 3)  # [M, P, H, G, d]
    z = (qg @ s["k"].float().transpose(-1, -2)) * s["scale"]  # [M, P, H, G, rows]
    z = z.masked_fill(torch.arange(z.shape[-1], device=z.device) >= s["lens"][:, None, None, None], -math.inf)
    zog = zo.view(M, P, G, H, -1).transpose(2, 3)
    m = torch.maximum(z.amax(-1), zog.amax(-1))[..., None]
    p, po = (z - m).exp(), (zog - m).exp()
    out = p @ s["v"].float()
    out += (po.transpose(2, 3).reshape(M, P * G, H, 1, -1) @ s["vo"].float()).view(M, P, G, H, d).transpose(2, 3)
    out /= (p.sum(-1) + po.sum(-1))[..., None]
    return {"out": out.transpose(2, 3).reshape(M, P * G, H, d)}


# ------------------------------------------------------------------------------------------
# 64 bits, from the definitions
# ------------------------------------------------------------------------------------------

def _turned(q, pos, rot):
    """One vector of complex pairs (column i with column i + rot / 2) turned by its angles."""
    q = q.double()
    if not rot:
        return q
    half = rot // 2
    angle = torch.tensor([float(pos) / _ROPE_BASE ** (2.0 * i / rot) for i in range(half)], dtype=torch.float64, device=q.device)
    z = torch.complex(q[..., :half].contiguous(), q[..., half:rot].contiguous()) * torch.polar(torch.ones_like(angle), angle)
    return torch.cat([z.real, z.imag, q[..., rot:]], -1)


def exact(case, seed):
    c = _case(case)
    w = work(case)
    x = _inputs(c, seed)
    H, d, scale = c["H"], c["d"], 1.0 / math.sqrt(c["d"])
    if c["kind"] == "scored":
        lens = _lens(c, c["b"])
        out = torch.zeros(c["M"], c["b"], H, d, dtype=torch.float64, device=DEVICE)
        scores = torch.zeros(c["M"], c["b"], H, max(lens), dtype=torch.float64, device=DEVICE)
        if c["M"] * c["b"] > 4000:
            return None
        for s, (n, hidden) in enumerate(zip(lens, _open_rows(c, lens))):
            rows = [i for i in range(n) if i != hidden]
            for m in range(c["M"]):
                q = _turned(x["q"][m, s], n - 1 - (hidden >= 0), c["rot"])
                z = torch.einsum("hd,hnd->hn", q, x["k"][m, s, :, rows].double()) * scale
                p = torch.softmax(z, -1)
                out[m, s] = torch.einsum("hn,hnd->hd", p, x["v"][m, s, :, rows].double())
                scores[m, s][:, rows] = p
        return {"out": out, "scores": scores}
    if c["kind"] == "prompt":
        if w["flops"] > 8e10 or sum(min(c["nq"], n) for n in _lens(c, c["b"])) > 40000:
            return None
        lens = _lens(c, c["b"])
        scores = torch.zeros(1, c["b"], H, max(lens), dtype=torch.float64, device=DEVICE)
        t = 0
        for s, n in enumerate(lens):
            kinds = _span_kinds(n, c["interior"])
            pos, hid = _tied_positions(kinds), torch.tensor(_hid(kinds), device=DEVICE)
            nq = min(c["nq"], n)
            k = x["k"][0, s, :, :n].double()
            i = torch.arange(n, device=DEVICE)
            for a in range(n - nq, n, 512):
                e = min(a + 512, n)
                q = torch.stack([_turned(x["q"][t + j - (n - nq)], pos[j], c["rot"]) for j in range(a, e)], 1)  # [H, e - a, d]
                at = torch.arange(a, e, device=DEVICE)[:, None]
                seen = (i <= at) & (at <= hid)
                for j in range(a, e):
                    if kinds[j] == CL:
                        seen[j - a] = i == j
                z = torch.einsum("hqd,hnd->hqn", q, k) * scale
                scores[0, s, :, :n] += torch.softmax(torch.where(seen, z, -math.inf), -1).sum(1)
            t += nq
        return {"scores": scores}
    if c["kind"] == "evict":
        n, keep, recent = c["keep"] + c["blk"], c["keep"], c["recent"]
        if c["M"] * c["b"] * H * n > 3e7:
            return None
        f = x["fresh"].cpu().numpy().astype(np.float64).reshape(-1, n)
        kept, scores = np.zeros((f.shape[0], keep), np.int64), np.zeros(f.shape)
        for r, row in enumerate(f):
            order = sorted(range(n - recent), key=lambda i: (-row[i], i))
            stay = set(order[:keep - recent])
            spare = iter(sorted(i for i in stay if i >= keep - recent))
            kept[r] = [i if i in stay else next(spare) for i in range(keep - recent)] + list(range(n - recent, n))
            scores[r, :keep] = row[kept[r]]
        shape = (c["M"], c["b"], H)
        return {"k": None, "v": None, "scores": torch.tensor(scores).view(*shape, n), "kept": torch.tensor(kept, dtype=torch.int32).view(*shape, keep)}
    lens, lown = _lens(c, c["P"]), _own_lens(c)
    if c["M"] * c["P"] * c["G"] > 6000:
        return None
    out = torch.zeros(c["M"], c["P"] * c["G"], H, d, dtype=torch.float64, device=DEVICE)
    for m in range(c["M"]):
        for p, n in enumerate(lens):
            kp, vp = x["k"][m, p, :, :n].double(), x["v"][m, p, :, :n].double()
            for s in range(p * c["G"], (p + 1) * c["G"]):
                q = _turned(x["q"][m, s], n + lown[s] - 1, c["rot"])
                k = torch.cat([kp, x["ko"][m, s, :, :lown[s]].double()], 1)
                v = torch.cat([vp, x["vo"][m, s, :, :lown[s]].double()], 1)
                z = torch.softmax((k @ q[..., None])[..., 0] * scale, -1)
                out[m, s] = (z[:, None] @ v)[:, 0]
    return {"out": out}
