"""Infinities and NaN in queries and keys: what the scores of the rows get from them, against softmaxes in 64 bits.  A
query one of whose visible logits is not a number, or +infinity, has weights that are NaN at every row it sees, and adds
nothing to the rows it does not see."""
import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc

from _serving import collected  # noqa: F401
from _serving import RTOL, make, per_row, query, rotate, rows_of

pytestmark = pytest.mark.gpu

N, CL, CR = kvc.NORMAL, kvc.CL, kvc.CR
INF, NAN = float("inf"), float("nan")


def weights(cache, s, q, n_q, scale):
    """(seen [n_q, n], weights [H, n_q, n]) of the last n_q tokens of sequence s in layer 0; q: [n_q, H, d].  Rows that a
    query does not see are left out of its softmax and get 0.  A rotated query goes into the products in parts, of either
    sign or 0, so that at an infinite key its logit is NaN where it would be -infinity."""
    meta = cache.prefill_keys(s, n_q)
    n = meta.size
    i = torch.arange(n, device="cuda")
    t = i[n - n_q:, None]
    is_cl = torch.tensor((meta & 1).astype(bool), device="cuda")[n - n_q:, None]
    seen = torch.where(is_cl, i == t, (i <= t) & (t <= torch.tensor(meta >> 1, device="cuda")))
    pos = cache.masked_reference_layout(s)["stored_pos"]
    qq = torch.stack([rotate(q[j], pos[n - n_q + j], cache.rotary_dim) for j in range(n_q)], 1)
    k = rows_of(cache, s, n)[0][0].double()
    z = torch.einsum("hqd,hnd->hqn", qq, k) * scale
    if cache.rotary_dim:
        z.masked_fill_(torch.isinf(k).any(-1)[:, None], NAN)
    w = torch.zeros_like(z)
    for j in range(n_q):
        w[:, j, seen[j]] = torch.softmax(z[:, j, seen[j]], -1)
    return seen, w


def agree(got, ref, what=""):
    """NaN where the reference is, its values elsewhere (RTOL of themselves, as every weight summed here is)."""
    got, ref = got.double().cpu(), ref.double().cpu()
    bad = torch.isnan(ref)
    assert bad.any() and not bad.all(), what
    assert torch.equal(torch.isnan(got), bad), what
    assert float(((got - ref).abs() - RTOL * ref.abs())[~bad].max()) <= 1e-9, what


# windows of up to 16 queries, of up to 128, whole prompts
WINDOWS = [12, 90, 700]


@pytest.mark.parametrize("n_q", WINDOWS)
@pytest.mark.parametrize("d,dtype,rot", [(64, "f16", 0), (80, "bf16", 80), (128, "bf16", 0)])
def test_infinite_logit_of_a_prompt_query(n_q, d, dtype, rot):
    """One infinite component: the query's logits are infinities of both signs.  The last query, which sees every row, in
    head 0, and one in the middle in head 1; head 2 is untouched."""
    cache, g = make(1, 3, d, [700], dtype, rot, seed=n_q)
    cache.attach_scores()
    q = torch.empty(n_q, 3, d, dtype=cache.torch_dtype, device="cuda").normal_(0.0, 2.0, generator=g)
    q[-1, 0, d - 1] = INF
    cache.score_prompt(0, q, [n_q], d ** -0.5)
    got = per_row(cache, cache.scores, 0, 700)[0]
    ref = weights(cache, 0, q, n_q, d ** -0.5)[1].sum(1)
    assert torch.isnan(ref[0]).all() and torch.isfinite(ref[1:]).all()
    agree(got, ref)
    assert cache.device_status() == 0


def spanned(n, spans):
    """Token kinds with spans [cl, cr]."""
    kinds = np.zeros(n, np.uint8)
    for cl, cr in spans:
        kinds[cl], kinds[cr] = CL, CR
    return kinds


@pytest.mark.parametrize("n_q", WINDOWS)
@pytest.mark.parametrize("d,dtype,rot", [(64, "f16", 64), (80, "bf16", 80), (96, "bf16", 0), (128, "f16", 0)])
def test_prompt_queries_that_are_not_finite(n_q, d, dtype, rot):
    """NaN and infinities in queries and keys: later rows, freed spans' interiors and <CL> rows' own weights stay numbers.
    Heads: a NaN query; a NaN key that the last queries see; an infinite key in a span's interior, hidden from the
    queries past its <CR>; logits that are all -infinity."""
    kinds = spanned(700, [(100, 130), (300, 350), (650, 692)])
    cache, g = make(1, 5, d, [700], dtype, rot, kinds=[kinds], seed=n_q + d)
    cache.attach_scores()
    q = torch.empty(n_q, 5, d, dtype=cache.torch_dtype, device="cuda").normal_(0.0, 2.0, generator=g)
    k = rows_of(cache, 0, 700)[0][0]
    q[n_q // 2, 0, d - 1] = NAN
    q[-1, 0, 2] = NAN
    k[1, 694, 5] = NAN
    k[2, 660, 1] = INF
    k[3] = k[3].abs()
    q[n_q - 3, 3] = -INF
    cache.score_prompt(0, q, [n_q], d ** -0.5)
    seen, w = weights(cache, 0, q, n_q, d ** -0.5)
    ref = w.sum(1)
    got = per_row(cache, cache.scores, 0, 700)[0]
    assert torch.isnan(ref[:4]).any(1).all() and torch.isfinite(ref[:3]).any(1).all() and torch.isfinite(ref[4]).all()
    agree(got, ref)
    assert cache.device_status() == 0


@pytest.mark.parametrize("n_q", WINDOWS)
def test_several_sequences_one_of_them_not_finite(n_q):
    cache, g = make(1, 2, 64, [700, 90, 130], "f16", seed=4)
    cache.attach_scores()
    n = [n_q, min(n_q, 90), min(n_q, 130)]
    q = torch.empty(sum(n), 2, 64, dtype=torch.float16, device="cuda").normal_(0.0, 2.0, generator=g)
    q[n[0] + n[1] - 2, 1] = NAN  # of the second sequence
    cache.score_prompt(0, q, n, 0.125)
    at = 0
    for s, m in enumerate(n):
        rows = (700, 90, 130)[s]
        ref = weights(cache, s, q[at:at + m], m, 0.125)[1].sum(1)
        got = per_row(cache, cache.scores, s, rows)[0]
        if s == 1:
            agree(got, ref)
        else:
            assert torch.isfinite(got).all()
            assert float(((got.double() - ref).abs() - RTOL * ref.abs()).max()) <= 1e-9
        at += m


@pytest.mark.parametrize("n_q", WINDOWS + [128])
@pytest.mark.parametrize("d,dtype,rot", [(64, "f16", 0), (96, "bf16", 96), (128, "bf16", 0)])
def test_cl_queries_that_are_not_finite(n_q, d, dtype, rot):
    """A <CL> query's weight at its own row, the only one it sees, is 1 where its logit is finite, whatever the rows before
    it hold, and NaN where it is not.  Heads: the query; its key; a NaN key before it, in a span's interior; nothing."""
    spans = [(40, 70), (100, 127), (191, 250), (300, 350), (639, 660), (689, 690), (694, 697)]
    kinds = spanned(700, spans)
    cache, g = make(1, 4, d, [700], dtype, rot, kinds=[kinds], seed=n_q + d)
    cache.attach_scores()
    q = torch.empty(n_q, 4, d, dtype=cache.torch_dtype, device="cuda").normal_(0.0, 2.0, generator=g)
    k = rows_of(cache, 0, 700)[0][0]
    for cl, _ in spans[::2]:
        if cl >= 700 - n_q:
            q[cl - (700 - n_q), 0] = INF
    q[694 - (700 - n_q), 0, 1] = NAN
    k[1, 694, 3] = INF
    k[2, 110, 0] = NAN
    cache.score_prompt(0, q, [n_q], d ** -0.5)
    ref = weights(cache, 0, q, n_q, d ** -0.5)[1].sum(1)
    got = per_row(cache, cache.scores, 0, 700)[0]
    assert torch.isnan(ref[0]).sum() == sum(c >= 700 - n_q for c in {694} | {c for c, _ in spans[::2]})
    for h in range(4):
        if torch.isnan(ref[h]).any():
            agree(got[h], ref[h], f"head {h}")
        else:
            assert torch.isfinite(got[h]).all()
            assert float(((got[h].double() - ref[h]).abs() - RTOL * ref[h].abs()).max()) <= 1e-9
    assert cache.device_status() == 0


# few segments (a CTA or a cluster each), and thousands (a warp each)
@pytest.mark.parametrize("M,H", [(1, 4), (30, 90)])
@pytest.mark.parametrize("d,dtype", [(64, "f16"), (80, "bf16"), (128, "f16")])
def test_decode_queries_that_are_not_finite(M, H, d, dtype):
    """A step's weights: NaN at the rows that such a query sees, nothing at the hidden ones (a closed span that is not
    freed), other heads and sequences untouched."""
    kinds = [np.array([N] * 5 + [CL] + [N] * 150 + [CR, N, N], np.uint8), np.zeros(90, np.uint8)]
    cache, g = make(M, H, d, [159, 90], dtype, kinds=kinds, seed=H)
    sc = cache.attach_scores()
    q = query(cache, g)
    k = rows_of(cache, 0, 159)[0][0]
    q[0, 0, 0, 0] = NAN
    q[0, 0, 1, d - 1] = INF
    k[2, 157, 5] = NAN
    k[3, 30] = INF  # hidden
    cache.decode_attention_scored(q, d ** -0.5)
    assert (cache.last_decode_plan["mode"] == 2) == (M > 1)
    seen = torch.tensor([i for i in range(159) if not 5 <= i < 156], device="cuda")
    hidden = torch.arange(5, 156, device="cuda")
    got = per_row(cache, sc, 0, 159)
    assert torch.isnan(got[0, :3][:, seen]).all()
    assert torch.all(got[:, :, hidden] == 0)
    assert torch.isfinite(got[0, 3:]).all() and torch.isfinite(got[1:]).all()
    for x in (got[0, 3:][:, seen], got[1:][:, :, seen], per_row(cache, sc, 1, 90)):
        assert float((x.double().sum(-1) - 1).abs().max() if x.numel() else 0) <= 1e-5
    w = torch.softmax(torch.einsum("d,nd->n", q[0, 0, 3].double(), k[3][seen].double()) * d ** -0.5, -1)
    assert float(((got[0, 3][seen].double() - w).abs() - RTOL * w).max()) <= 1e-9


def test_long_segment_of_a_query_that_is_not_finite():
    """A cluster of CTAs, and rows past the logits that they hold."""
    n = 90000
    kinds = [np.array([N] * 40000 + [CL] + [N] * 45000 + [CR] + [N] * (n - 85002), np.uint8)]
    cache, g = make(1, 2, 64, [n], kinds=kinds, seed=9)
    sc = cache.attach_scores()
    q = query(cache, g)
    q[0, 0, 0, 7] = NAN
    cache.decode_attention_scored(q, 0.125)
    got = per_row(cache, sc, 0, n)[0]
    assert torch.all(got[:, 40000:85001] == 0)
    assert torch.isnan(got[0, :40000]).all() and torch.isnan(got[0, 85001:]).all()
    assert abs(float(got[1].double().sum()) - 1) <= 1e-5
    assert cache.device_status() == 0
