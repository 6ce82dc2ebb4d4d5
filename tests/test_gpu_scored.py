"""Decode attention that adds each row's weight to its score, against a plain 64-bit form."""
import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc

from _serving import collected  # noqa: F401
from _serving import attend, close, close_weights, make, per_row, query, rotate, rows_of

pytestmark = pytest.mark.gpu


def check(cache, q, scale, seen, qpos, before, out, n_layers=None, first=0):
    """seen[s]: the rows that the query of s sees; before: the scores before the call."""
    scores = cache.scores
    for s in range(cache.b):
        n = int(cache.capacity[s])
        added = per_row(cache, scores.double() - before.double(), s, n)
        k, v = rows_of(cache, s, n)
        for i in range(q.shape[0]):
            m = first + i
            if not len(seen[s]):
                assert torch.all(added[m] == 0)
                continue
            ref, w = attend(rotate(q[i, s], qpos[s], cache.rotary_dim), k[m], v[m], seen[s], scale)
            close(out[i, s], ref, f"out of sequence {s}, layer {m}")
            full = torch.zeros_like(added[m])
            full[:, seen[s]] = w
            if before.abs().max() == 0:
                close_weights(added[m], full, f"weights of sequence {s}, layer {m}")
            else:
                assert (added[m] - full).abs().max() <= 4e-7 * (1 + per_row(cache, scores, s, n)[m].abs().max())


LENS = [
    [1], [2], [3], [31], [33], [127], [128], [129], [257], [1000],
    [1, 0, 130, 64],            # a sequence without tokens
    [5000],                     # a cluster, several tiles each
    [4000, 3, 700, 65],         # unbalanced
]


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("d,dtype,rot", [(64, "f16", 0), (80, "bf16", 80), (96, "f16", 32), (128, "bf16", 0)])
def test_lengths(lens, d, dtype, rot):
    cache, g = make(2, 3, d, lens, dtype, rot, seed=sum(lens) + d)
    cache.attach_scores()
    before = cache.scores.clone()
    q = query(cache, g)
    scale = d ** -0.5
    out = cache.decode_attention_scored(q, scale)
    check(cache, q, scale, [list(range(n)) for n in lens], [n - 1 for n in lens], before, out)
    # the same attention as the decode's
    plain = cache.decode_attention_layers(q, scale)
    for s, n in enumerate(lens):
        if n:
            close(out[:, s], plain[:, s])
    assert cache.device_status() == 0


@pytest.mark.parametrize("M,H,b,n", [(24, 32, 2, 200), (6, 32, 16, 90), (3, 16, 32, 700), (1, 40, 8, 2500)])
def test_many_segments(M, H, b, n):
    """Several segments per CTA, a CTA each, and more CTAs than a wave."""
    cache, g = make(M, H, 64, [n] * b, seed=n)
    cache.attach_scores()
    before = cache.scores.clone()
    q = query(cache, g)
    out = cache.decode_attention_scored(q, 0.125)
    check(cache, q, 0.125, [list(range(n))] * b, [n - 1] * b, before, out)


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16")])
def test_rows_past_the_logits_in_shared_memory(d, dtype):
    """More rows than eight CTAs hold the logits of: the rest are computed a second time."""
    n = 120001
    cache, g = make(1, 1, d, [n], dtype, seed=5)
    cache.attach_scores()
    before = cache.scores.clone()
    q = query(cache, g)
    out = cache.decode_attention_scored(q, d ** -0.5)
    check(cache, q, d ** -0.5, [list(range(n))], [n - 1], before, out)


@pytest.mark.parametrize("policy", [kvc.POLICY_PAPER, kvc.POLICY_KEEP_CL])
def test_hidden_rows_get_nothing(policy):
    N, CL, CR = kvc.NORMAL, kvc.CL, kvc.CR
    kinds = [np.array([N] * 70 + [CL] + [N] * 9, np.uint8),       # an open span: its <CL> is hidden (paper)
             np.array([N] * 40 + [CL], np.uint8),                 # a <CL> query: itself alone
             np.array([N] * 5 + [CL] + [N] * 150 + [CR], np.uint8),        # a <CR> query sees its interior
             np.array([N] * 5 + [CL] + [N] * 150 + [CR, N, N], np.uint8),  # a closed span, not freed: one hidden run
             np.array([CL], np.uint8)]
    lens = [k.size for k in kinds]
    cache, g = make(2, 2, 64, lens, kinds=kinds, policy=policy)
    cache.attach_scores()
    before = cache.scores.clone()
    q = query(cache, g)
    out = cache.decode_attention_scored(q, 0.125)
    paper = policy == kvc.POLICY_PAPER
    seen = [[i for i in range(80) if i != 70 or not paper], [40],
            [i for i in range(157) if i != 5 or not paper],
            [i for i in range(159) if not (5 < i < 156 or (i == 5 and paper))], [0]]
    check(cache, q, 0.125, seen, [0] * 5, before, out)


@pytest.mark.parametrize("d,dtype,rot", [(64, "f16", 0), (64, "bf16", 64), (80, "f16", 48), (80, "bf16", 0), (96, "bf16", 96),
                                         (96, "f16", 0), (128, "f16", 128), (128, "bf16", 0)])
def test_thousands_of_short_segments(d, dtype, rot):
    """A warp for each segment, of one row up to as many as a warp holds the logits of; hidden runs, <CL> queries, a
    sequence without tokens; twice, so that the second call adds to the first's."""
    N, CL, CR = kvc.NORMAL, kvc.CL, kvc.CR
    kinds = [np.array([N] * n, np.uint8) for n in (1, 2, 0, 31, 32, 33, 127, 129, 1023)] + [
        np.array([N] * 70 + [CL] + [N] * 9, np.uint8),
        np.array([N] * 40 + [CL], np.uint8),
        np.array([N] * 5 + [CL] + [N] * 150 + [CR], np.uint8),
        np.array([N] * 5 + [CL] + [N] * 150 + [CR, N, N], np.uint8),
        np.array([CL], np.uint8)]
    seen = [list(range(k.size)) for k in kinds[:9]] + [
        [i for i in range(80) if i != 70], [40], [i for i in range(157) if i != 5], [i for i in range(159) if not 5 <= i < 156], [0]]
    lens = [k.size for k in kinds]
    cache, g = make(12, 16, d, lens, dtype, rot, kinds=kinds, seed=d + rot, spare=3)
    cache.attach_scores()
    q = query(cache, g)
    plain = cache.decode_attention_layers(q, d ** -0.5)
    qpos = [cache.masked_reference_layout(s)["pos"][-1] if n else 0 for s, n in enumerate(lens)]
    for _ in range(2):
        before = cache.scores.clone()
        out = cache.decode_attention_scored(q, d ** -0.5)
        check(cache, q, d ** -0.5, seen, qpos, before, out)
        assert cache.last_decode_plan["mode"] == 2
    for s, n in enumerate(lens):
        if n:
            close(out[:, s], plain[:, s])
    again = [cache.scores.clone(), out]
    cache.attach_scores()
    cache.decode_attention_scored(q, d ** -0.5)
    out = cache.decode_attention_scored(q, d ** -0.5)
    assert torch.equal(again[0], cache.scores) and torch.equal(again[1][:, lens.index(1)], out[:, lens.index(1)])


def test_scores_add_up_over_steps_and_layers_by_turns():
    cache, g = make(3, 4, 64, [100, 37], spare=8)
    cache.attach_scores()
    for step in range(5):
        new = torch.empty(3, 2, 4, 64, dtype=torch.float16, device="cuda").normal_(generator=g)
        cache.append(new, new, [1, 1], [0, 0])
        q = query(cache, g)
        before = cache.scores.clone()
        seen = [list(range(101 + step)), list(range(38 + step))]
        if step % 2:
            out = cache.decode_attention_scored(q, 0.125)
            check(cache, q, 0.125, seen, [0, 0], before, out)
        else:
            for first, n in ((1, 2), (0, 1)):
                before = cache.scores.clone()
                part = q[first:first + n].contiguous()
                out = cache.decode_attention_scored(part, 0.125, first=first, n_layers=n)
                check(cache, part, 0.125, seen, [0, 0], before, out, first=first)
    total = cache.scores.double().view(3, -1).sum(1)
    assert torch.allclose(total, torch.full_like(total, 5 * 2 * 4.0), rtol=1e-5)


def test_the_same_bits_every_time():
    cache, g = make(2, 8, 80, [3000, 50, 700], "bf16", 80)
    q = query(cache, g)
    runs = []
    for _ in range(3):
        cache.attach_scores()
        runs.append((cache.decode_attention_scored(q, 0.1), cache.scores.clone()))
    for out, sc in runs[1:]:
        assert torch.equal(out, runs[0][0]) and torch.equal(sc, runs[0][1])


def test_rows_beyond_a_sequence_are_not_read():
    cache, g = make(1, 2, 64, [200, 33], spare=90)
    ref = cache.k.clone(), cache.v.clone()
    for s, n in enumerate((200, 33)):
        for plane in (cache.k, cache.v):
            base, cap = cache.H * int(cache.offsets[s]), int(cache.capacity[s])
            plane.view(-1, 64)[base:base + 2 * cap].view(2, cap, 64)[:, n:] = float("nan")
    cache.attach_scores()
    q = query(cache, g)
    out = cache.decode_attention_scored(q, 0.125)
    check(cache, q, 0.125, [list(range(200)), list(range(33))], [0, 0], torch.zeros_like(cache.scores), out)
    del ref


def test_compaction_moves_scores_with_their_rows():
    N, CL, CR = kvc.NORMAL, kvc.CL, kvc.CR
    rng = np.random.default_rng(3)
    kinds, spans = [], []
    for s in range(3):
        k = []
        for _ in range(int(rng.integers(1, 30))):
            k += [N] * int(rng.integers(0, 90)) + [CL] + [N] * int(rng.integers(0, 70)) + [CR]
        k += [N] * 5
        kinds.append(np.array(k, np.uint8))
    lens = [k.size for k in kinds]
    cache, g = make(2, 3, 64, lens, kinds=kinds)
    sc = cache.attach_scores()
    for s, n in enumerate(lens):
        per_row(cache, sc, s, n).copy_(torch.rand(2, 3, n, device="cuda"))
    old = [per_row(cache, sc, s, n).clone() for s, n in enumerate(lens)]
    for s in (0, 2):
        for cl, cr in cache.pending_spans(s):
            spans.append((s, cl, cr))
    cache.compress_spans(*map(list, zip(*spans)))
    for s, n in enumerate(lens):
        rows = cache.masked_reference_layout(s)["stored_orig"]
        new = per_row(cache, cache.scores, s, n)
        assert torch.equal(new[:, :, :rows.size], old[s][:, :, torch.tensor(rows, device="cuda", dtype=torch.long)])
        assert torch.all(new[:, :, rows.size:] == 0)


def test_on_another_stream():
    cache, g = make(2, 4, 64, [500, 900])
    cache.attach_scores()
    q = query(cache, g)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = torch.empty(2, 2, 4, 64, device="cuda")
    cache.decode_attention_scored(q, 0.125, out=out, stream=side)
    side.synchronize()
    check(cache, q, 0.125, [list(range(500)), list(range(900))], [0, 0], torch.zeros_like(cache.scores), out)


def test_refusals():
    cache, g = make(2, 2, 64, [10])
    q = query(cache, g)
    with pytest.raises(kvc.KvcError) as e:
        cache.decode_attention_scored(q, 0.125)
    assert e.value.status == 5  # no scores
    cache.attach_scores()
    with pytest.raises(kvc.KvcError) as e:
        cache.decode_attention_scored(q, float("nan"))
    assert e.value.status == 1
    with pytest.raises(kvc.KvcError) as e:
        cache.decode_attention_scored(q, 0.125, first=1, n_layers=2)
    assert e.value.status == 1
    with pytest.raises(ValueError):
        cache.decode_attention_scored(q.float(), 0.125)
    with pytest.raises(ValueError):
        cache.attach_scores(torch.zeros(7, device="cuda"))
    with pytest.raises(kvc.KvcError) as e:
        kvc.kvc_set_scores(cache.handle, torch.zeros(2 * 2 * 10 + 1, device="cuda")[1:])
    assert e.value.status == 1
    new = torch.zeros(1, 2, 64, dtype=torch.float16, device="cuda")
    cache2, _ = make(2, 2, 64, [10], spare=2)
    cache2.attach_scores()
    cache2.append(new, new, [1], [0], layer=0)
    with pytest.raises(kvc.KvcError) as e:  # layer 1 is not written
        cache2.decode_attention_scored(q, 0.125)
    assert e.value.status == 5
    local = kvc.KVCache(1, 2, 64, [64], policy=kvc.POLICY_LOCAL, local_ratio=0.5)
    with pytest.raises(kvc.KvcError) as e:
        local.attach_scores()
    assert e.value.status == 2
    assert torch.all(cache.scores == 0)


@pytest.mark.parametrize("M,H,lens,mode", [(12, 16, [1, 2, 31, 33, 129, 1023, 400, 90, 700, 64, 5, 300, 12], 2), (2, 8, [3000, 50, 700], 4),
                                           (1, 4, [5000], 1), (24, 16, [200, 200], 1)])
def test_outputs_and_scores_repeat_bit_for_bit(M, H, lens, mode):
    """Every sequence's, in a warp, a CTA or a cluster per segment; also where the scores are added to what is there."""
    cache, g = make(M, H, 80, lens, "bf16", 80, seed=M)
    q = query(cache, g)
    runs = []
    for _ in range(3):
        cache.attach_scores()
        a = cache.decode_attention_scored(q, 0.1)
        assert cache.last_decode_plan["mode"] == mode
        b = cache.decode_attention_scored(q, 0.1)
        runs.append((a, b, cache.scores.clone()))
    for run in runs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(run, runs[0]))
    assert torch.equal(runs[0][0], runs[0][1])
