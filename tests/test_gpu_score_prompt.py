"""Attention weights of a prompt's queries added to its rows' scores, against a plain 64-bit form."""
import numpy as np
import pytest
import torch

import oracle as orc
import paper_2310_08152_gb300 as kvc

from _serving import collected  # noqa: F401
from _serving import close_weights, make, per_row, rotate, rows_of

pytestmark = pytest.mark.gpu

N, CL, CR = kvc.NORMAL, kvc.CL, kvc.CR


def queries(cache, n_q, g, sd=2.0):
    return torch.empty(sum(n_q), cache.H, cache.d, dtype=cache.torch_dtype, device="cuda").normal_(0.0, sd, generator=g)


def reference(cache, layer, s, q, n_q, scale, pos):
    """Summed weights [H, rows] of the last n_q tokens, from the mask bounds of the span book."""
    meta = cache.prefill_keys(s, n_q)
    n = meta.size
    hid, is_cl = torch.tensor(meta >> 1, device="cuda"), meta & 1
    k = rows_of(cache, s, n)[0][layer].double()
    total = torch.zeros(cache.H, n, dtype=torch.float64, device="cuda")
    i = torch.arange(n, device="cuda")
    for a in range(n - n_q, n, 256):
        e = min(a + 256, n)
        qq = torch.stack([rotate(q[j - (n - n_q)], pos[j], cache.rotary_dim) for j in range(a, e)], 1)
        t = torch.arange(a, e, device="cuda")[:, None]
        seen = (i <= t) & (t <= hid)
        for j in range(a, e):
            if is_cl[j]:
                seen[j - a] = i == j
        z = torch.einsum("hqd,hnd->hqn", qq, k) * scale
        total += torch.softmax(z.masked_fill(~seen, -torch.inf), -1).sum(1)
    return total


def check(cache, n_q, g, layer=0, scale=None, sd=2.0):
    scale = cache.d ** -0.5 if scale is None else scale
    q = queries(cache, n_q, g, sd)
    cache.attach_scores()
    cache.score_prompt(layer, q, n_q, scale)
    at = 0
    for s in range(cache.b):
        n = int(cache.lengths()[0][s])
        got = per_row(cache, cache.scores, s, int(cache.capacity[s]))
        for m in range(cache.M):
            if m != layer or n_q[s] == 0:
                assert torch.all(got[m] == 0), (s, m)
        assert torch.all(got[:, :, n:] == 0)
        if n_q[s]:
            pos = cache.masked_reference_layout(s)["stored_pos"]
            ref = reference(cache, layer, s, q[at:at + n_q[s]], n_q[s], scale, pos)
            close_weights(got[layer, :, :n], ref, f"sequence {s}")
        at += n_q[s]
    assert cache.device_status() == 0


CASES = [([1], [1]), ([2], [1]), ([5], [5]), ([127], [127]), ([128], [128]), ([129], [129]), ([130], [1]), ([257], [128]),
         ([300], [300]), ([1000], [17]), ([1000], [16]), ([777, 30, 4], [9, 16, 1]), ([500], [80]), ([1000], [641]), ([40, 700, 128, 3], [40, 100, 0, 3]), ([600, 90, 1], [500, 0, 1])]


@pytest.mark.parametrize("lens,n_q", CASES, ids=lambda x: str(x))
@pytest.mark.parametrize("d,dtype,rot", [(64, "f16", 0), (64, "bf16", 64), (80, "bf16", 0), (80, "f16", 80), (96, "f16", 32),
                                         (96, "bf16", 0), (128, "bf16", 128), (128, "f16", 0)])
def test_lengths(lens, n_q, d, dtype, rot):
    cache, g = make(2, 2, d, lens, dtype, rot, seed=sum(lens))
    check(cache, n_q, g, layer=1)


@pytest.mark.parametrize("d,dtype,rot", [(64, "f16", 0), (128, "bf16", 128)])
def test_long_prompt(d, dtype, rot):
    cache, g = make(1, 1, d, [5003], dtype, rot, seed=1)
    check(cache, [5003], g)
    check(cache, [33], g)
    cache, g = make(1, 8, d, [20011, 40], dtype, rot, seed=2)
    check(cache, [64, 40], g)
    check(cache, [11, 16], g)


@pytest.mark.parametrize("H,lens,n_q", [(32, [2048, 1500], [2048, 700]), (40, [900] * 12, [900] * 12), (32, [3000] * 8, [100] * 8)])
def test_many_units(H, lens, n_q):
    cache, g = make(1, H, 64, lens, "bf16")
    check(cache, n_q, g)


def spans(rng, n):
    k = []
    while len(k) < n:
        k += [N] * int(rng.integers(0, 70)) + [CL] + [N] * int(rng.integers(0, 150)) + [CR]
    return np.array(k[:n], np.uint8)


@pytest.mark.parametrize("policy", [kvc.POLICY_PAPER, kvc.POLICY_KEEP_CL])
@pytest.mark.parametrize("rot", [0, 64])
def test_masks(policy, rot):
    rng = np.random.default_rng(5 + policy)
    kinds = [spans(rng, n) for n in (1000, 411, 128, 130, 700)]
    lens = [k.size for k in kinds]
    cache, g = make(1, 2, 64, lens, rot=rot, kinds=kinds, policy=policy)
    check(cache, lens, g)
    check(cache, [200, 128, 1, 129, 300], g)
    check(cache, [100, 128, 1, 77, 30], g)
    check(cache, [16, 3, 1, 16, 12], g)


def test_bounds_agree_with_the_oracle():
    """The mask bounds that the reference here reads are the oracle's visibility."""
    rng = np.random.default_rng(9)
    kinds = spans(rng, 300)
    cache, _ = make(1, 1, 64, [300], kinds=[kinds])
    meta = cache.prefill_keys(0, 300)
    for t in range(300):
        vis = orc.visible(kinds, t, orc.POLICY_PAPER)[:t + 1]
        mine = [i == t if meta[t] & 1 else i <= t <= (meta[i] >> 1) for i in range(t + 1)]
        assert list(map(bool, vis)) == mine, t


def test_only_sentinels():
    cache, g = make(1, 2, 64, [260], kinds=[np.array([CL, CR] * 130, np.uint8)])
    check(cache, [260], g)
    check(cache, [100], g)
    check(cache, [16], g)
    check(cache, [1], g)


def test_large_logits_and_small_scales():
    for scale, sd in ((4.0, 4.0), (1e-5, 1.0)):
        cache, g = make(1, 2, 64, [500])
        q = queries(cache, [500], g, sd)
        cache.attach_scores()
        cache.score_prompt(0, q, [500], scale)
        ref = reference(cache, 0, 0, q, 500, scale, np.zeros(500))
        got = per_row(cache, cache.scores, 0, 500)[0].double()
        # a logit of 2^8 and more in 32 bits: the weights of close ones move by its last bits
        assert float((got - ref).norm() / ref.norm()) <= (2e-3 if scale > 1 else 2e-5)
        assert abs(float(got.sum()) - 1000.0) <= 1e-2


def test_rows_past_the_end_are_masked():
    cache, g = make(2, 2, 64, [200, 150], spare=60)
    for plane in (cache.k, cache.v):
        for s, n in enumerate((200, 150)):
            base, cap = 2 * int(cache.offsets[s]), int(cache.capacity[s])
            for m in range(2):
                plane.view(2, -1, 64)[m, base:base + 2 * cap].view(2, cap, 64)[:, n:] = float("nan")
    check(cache, [200, 40], g, layer=1)


def test_adds_to_what_is_there_and_repeats_bit_for_bit():
    cache, g = make(1, 4, 80, [700], "bf16", 80)
    q = queries(cache, [700], g)
    cache.attach_scores()
    cache.score_prompt(0, q, [700], 0.11)
    once = cache.scores.clone()
    for _ in range(3):
        cache.attach_scores()
        cache.score_prompt(0, q, [700], 0.11)
        assert torch.equal(cache.scores, once)
    cache.score_prompt(0, q, [700], 0.11)
    assert torch.equal(cache.scores, once + once)
    # the sums are those of the tokens' decodes
    assert abs(float(once.double().sum()) - 4 * 700) <= 1e-2


def test_block_by_block_with_freeing_and_eviction():
    """A prompt in blocks as the paper's loop runs it: append, score, free the closed spans, evict; on a side stream."""
    rng = np.random.default_rng(2)
    kinds = spans(rng, 900)
    cache = kvc.KVCache(2, 3, 64, [900])
    cache.attach_scores()
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for a in range(0, 900, 180):
            kv = torch.empty(2, 2, 180, 3, 64, dtype=torch.float16, device="cuda").normal_(generator=g)
            cache.append(kv[0], kv[1], [180], kinds[a:a + 180])
            for m in range(2):
                q = queries(cache, [180], g)
                before = per_row(cache, cache.scores, 0, 900)[m].clone()
                cache.score_prompt(m, q, [180], 0.125)
                n = int(cache.lengths()[0][0])
                ref = reference(cache, m, 0, q, 180, 0.125, np.zeros(n))
                got = per_row(cache, cache.scores, 0, 900)[m]
                side.synchronize()
                assert float((got.double() - before.double())[:, :n].sub(ref).abs().max()) <= 2e-5 * (1 + float(got.max()))
            done = cache.pending_spans(0)
            if done:
                cache.compress_spans([0] * len(done), *map(list, zip(*done)))
            if int(cache.lengths()[0][0]) > 260 and kinds[:a + 180].tolist().count(CL) == kinds[:a + 180].tolist().count(CR):
                cache.evict(260, 60)
    assert cache.device_status() == 0


def test_refusals():
    cache, g = make(2, 2, 64, [50], spare=5)
    q = queries(cache, [50], g)
    with pytest.raises(kvc.KvcError) as e:
        cache.score_prompt(0, q, [50], 0.125)
    assert e.value.status == 5  # no scores
    cache.attach_scores()
    for bad in (0.0, -1.0, float("inf")):
        with pytest.raises(kvc.KvcError) as e:
            cache.score_prompt(0, q, [50], bad)
        assert e.value.status == 1
    with pytest.raises(kvc.KvcError) as e:
        cache.score_prompt(2, q, [50], 0.125)
    assert e.value.status == 1
    with pytest.raises(ValueError):
        cache.score_prompt(0, q, [49], 0.125)
    with pytest.raises(ValueError):
        cache.score_prompt(0, q, [25, 25], 0.125)
    with pytest.raises(kvc.KvcError) as e:
        cache.score_prompt(0, torch.zeros(51, 2, 64, dtype=torch.float16, device="cuda"), [51], 0.125)
    assert e.value.status == 1
    with pytest.raises(kvc.KvcError) as e:
        kvc.kvc_score_prompt(cache.handle, 0, q, [50], 0.125, torch.zeros(8, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 1
    cache.score_prompt(0, q[:0], [0], 0.125)  # nothing to do
    new = torch.zeros(1, 2, 64, dtype=torch.float16, device="cuda")
    cache.append(new, new, [1], [0], layer=0)
    with pytest.raises(kvc.KvcError) as e:  # layer 1 is not written
        cache.score_prompt(1, q, [50], 0.125)
    assert e.value.status == 5
    kinds = np.array([N, CL, N, CR, N], np.uint8)
    freed = kvc.KVCache(1, 2, 64, [8])
    kv = torch.zeros(1, 5, 2, 64, dtype=torch.float16, device="cuda")
    freed.append(kv, kv, [5], kinds, free_closed=True)
    freed.attach_scores()
    with pytest.raises(kvc.KvcError) as e:  # a query token is not stored
        freed.score_prompt(0, kv[0], [5], 0.125)
    assert e.value.status == 5
    assert torch.all(cache.scores == 0)
