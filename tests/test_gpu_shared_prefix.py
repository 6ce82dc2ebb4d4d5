"""Decode attention of sequences that share a prefix, against a plain 64-bit form."""
import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc

from _serving import collected  # noqa: F401
from _serving import attend, close, make, query, rotate, rows_of

pytestmark = pytest.mark.gpu


def pair(M, H, d, lens, parent, own, dtype="f16", rot=0, seed=0, spare=0, kinds=None):
    prefix, _ = make(M, H, d, lens, dtype, rot, seed=seed, spare=spare)
    pos = np.concatenate([(lens[p] if p >= 0 else 0) + np.arange(n) for p, n in zip(parent, own)] + [np.zeros(0, np.int64)])
    cache, g = make(M, H, d, own, dtype, rot, seed=seed + 1, spare=spare, pos=pos.astype(np.int32), kinds=kinds)
    cache.set_prefix(prefix, parent)
    return prefix, cache, g


def check(prefix, cache, parent, own, q, scale, out, seen=None, first=0, cl=()):
    plen = prefix.lengths()[0]
    for s in range(cache.b):
        if own[s] == 0:
            continue
        n = int(plen[parent[s]]) if parent[s] >= 0 and s not in cl else 0
        ko, vo = rows_of(cache, s, own[s])
        rows = torch.tensor(list(range(own[s])) if seen is None else seen[s], device="cuda")
        k, v = ko[:, :, rows], vo[:, :, rows]
        if n:
            kp, vp = rows_of(prefix, parent[s], n)
            k, v = torch.cat([kp, k], 2), torch.cat([vp, v], 2)
        qpos = (int(plen[parent[s]]) if parent[s] >= 0 else 0) + own[s] - 1
        for i in range(q.shape[0]):
            ref, _ = attend(rotate(q[i, s], qpos, cache.rotary_dim), k[first + i], v[first + i], list(range(k.shape[2])), scale)
            close(out[i, s], ref, f"sequence {s}, layer {first + i}")


GROUPS = [
    ([1], [0], [1]),
    ([5], [0, 0], [1, 3]),
    ([63], [0] * 8, [1, 2, 3, 4, 5, 6, 7, 8]),
    ([64], [0] * 9, [9] * 9),
    ([65], [0] * 16, [4] * 16),
    ([200], [0] * 17, [3] * 17),
    ([257, 33], [0, 1] * 16, [5] * 32),
    ([1000], [0] * 33, [2] * 33),
    ([700, 1, 90], [0] * 64 + [1] * 3 + [-1] + [2] * 65, [1 + i % 7 for i in range(133)]),
    ([5000], [0] * 3, [300, 1, 40]),
    ([300, 0, 40], [0, 1, 2, -1, 1], [4, 5, 0, 7, 1]),   # an empty prefix, no prefix, no own rows
]


@pytest.mark.parametrize("lens,parent,own", GROUPS, ids=lambda x: str(x)[:24])
@pytest.mark.parametrize("d,dtype,rot", [(64, "f16", 0), (80, "f16", 80), (80, "bf16", 32), (96, "bf16", 0), (128, "bf16", 128),
                                         (128, "f16", 0)])
def test_groups(lens, parent, own, d, dtype, rot):
    prefix, cache, g = pair(2, 2, d, lens, parent, own, dtype, rot, seed=len(parent))
    q = query(cache, g)
    out = cache.decode_attention_shared(q, d ** -0.5, out=torch.full(q.shape, 7.0, device="cuda"))
    check(prefix, cache, parent, own, q, d ** -0.5, out)
    for s, n in enumerate(own):
        if n == 0:
            assert torch.all(out[:, s] == 7.0)  # skipped
    assert cache.device_status() == 0 and prefix.device_status() == 0


@pytest.mark.parametrize("n,members", [(40000, 2), (9001, 64), (3000, 130)])
@pytest.mark.parametrize("d,dtype", [(64, "f16"), (128, "bf16")])
def test_long_prefixes_are_split(n, members, d, dtype):
    prefix, cache, g = pair(1, 1, d, [n], [0] * members, [1 + i % 3 for i in range(members)], dtype, seed=n)
    q = query(cache, g)
    out = cache.decode_attention_shared(q, d ** -0.5)
    check(prefix, cache, [0] * members, [1 + i % 3 for i in range(members)], q, d ** -0.5, out)


@pytest.mark.parametrize("dtype,rising", [("f16", False), ("bf16", True), ("f16", True)])
def test_runs_of_several_sums(dtype, rising):
    """Enough heads and layers that a long prefix is not split: its sums go to memory now and then, with a maximum that stays
    or that keeps growing between them."""
    parent, own = [0] * 40, [1 + i % 2 for i in range(40)]
    prefix, cache, g = pair(19, 32, 64, [5000], parent, own, dtype)
    if rising:
        prefix.k.view(19, 32, 5000, 64).mul_(torch.linspace(0.2, 4.0, 5000, device="cuda")[:, None].to(prefix.k.dtype))
    q = query(cache, g)
    out = cache.decode_attention_shared(q, 0.25 if rising else 0.125)
    kp, vp = rows_of(prefix, 0, 5000)
    for m, h, s in ((0, 0, 0), (3, 31, 39), (18, 5, 17), (9, 16, 2)):
        ko, vo = rows_of(cache, s, own[s])
        k, v = torch.cat([kp[m, h:h + 1], ko[m, h:h + 1]], 1), torch.cat([vp[m, h:h + 1], vo[m, h:h + 1]], 1)
        ref, _ = attend(q[m, s, h:h + 1].double(), k, v, list(range(k.shape[1])), 0.25 if rising else 0.125)
        close(out[m, s, h:h + 1], ref, f"layer {m}, head {h}, sequence {s}")
    assert cache.device_status() == 0


def test_many_layers_and_part_of_them():
    parent, own = [0, 0, 1, 1, 1], [3, 4, 5, 6, 70]
    prefix, cache, g = pair(12, 16, 64, [500, 130], parent, own)
    q = query(cache, g)
    out = cache.decode_attention_shared(q, 0.125)
    check(prefix, cache, parent, own, q, 0.125, out)
    part = q[3:5].contiguous()
    out2 = cache.decode_attention_shared(part, 0.125, first=3, n_layers=2)
    check(prefix, cache, parent, own, part, 0.125, out2, first=3)
    one = cache.decode_attention_shared(q[11:].contiguous(), 0.125, first=11)
    check(prefix, cache, parent, own, q[11:], 0.125, one, first=11)


def test_large_and_equal_logits():
    """A running maximum that keeps growing, one that never does, and logits that are all the same."""
    for scale in (8.0, -2.0, 0.0, 1e-6):
        prefix, cache, g = pair(1, 2, 64, [1500], [0] * 5, [2] * 5)
        if scale == 8.0:
            ramp = torch.linspace(-1, 1, 1500, device="cuda").half()
            k, _ = rows_of(prefix, 0, 1500)
            k.copy_(ramp[None, None, :, None].expand_as(k))
        q = query(cache, g)
        out = cache.decode_attention_shared(q, scale)
        check(prefix, cache, [0] * 5, [2] * 5, q, scale, out)


def test_own_rows_hidden_and_cl_queries():
    N, CL, CR = kvc.NORMAL, kvc.CL, kvc.CR
    kinds = [np.array([N, N, CL, N], np.uint8), np.array([CL], np.uint8), np.array([N, CL], np.uint8),
             np.array([CL, N, N, CR], np.uint8)]
    own = [4, 1, 2, 4]
    prefix, cache, g = pair(2, 2, 64, [100], [0] * 4, own, kinds=kinds)
    q = query(cache, g)
    out = cache.decode_attention_shared(q, 0.125)
    check(prefix, cache, [0] * 4, own, q, 0.125, out, seen=[[0, 1, 3], [0], [1], [1, 2, 3]], cl=(1, 2))


def test_one_sequence_of_a_group_does_not_touch_another():
    """A query with infinities or NaN spoils its own output only; rows past the prefix's end are not read."""
    parent, own = [0] * 6, [3] * 6
    prefix, cache, g = pair(1, 2, 64, [150], parent, own, spare=70)
    for c, n in ((prefix, 150), (cache, 3)):
        for plane in (c.k, c.v):
            for s in range(c.b):
                base, cap = c.H * int(c.offsets[s]), int(c.capacity[s])
                plane.view(-1, 64)[base:base + 2 * cap].view(2, cap, 64)[:, n:] = float("nan")
    q = query(cache, g)
    clean = cache.decode_attention_shared(q, 0.125)
    check(prefix, cache, parent, own, q, 0.125, clean)
    bad = q.clone()
    bad[0, 2, 0, 5], bad[0, 4, 1, 0] = float("nan"), float("inf")
    out = cache.decode_attention_shared(bad, 0.125)
    for s in range(6):
        for h in range(2):
            if (s, h) in ((2, 0), (4, 1)):
                assert torch.isnan(out[0, s, h]).all()
            else:
                assert torch.equal(out[0, s, h], clean[0, s, h])


def test_prefix_and_own_rows_change_between_calls():
    """Own tokens are appended, the prefix grows, is evicted and compacted; the parents change."""
    parent, own = [0, 0, 1, 1], [1, 1, 1, 1]
    prefix, cache, g = pair(2, 3, 64, [300, 200], parent, own, spare=40)
    prefix.attach_scores(torch.rand(2, 3 * prefix.C, device="cuda"))
    for s, n in enumerate((300, 200)):
        base, cap = 3 * int(prefix.offsets[s]), int(prefix.capacity[s])
        prefix.scores.view(2, -1)[:, base:base + 3 * cap].view(2, 3, cap)[:, :, n:] = 0

    def step():
        new = torch.empty(2, 4, 3, 64, dtype=torch.float16, device="cuda").normal_(generator=g)
        cache.append(new, new, [1] * 4, [0] * 4)
        for s in range(4):
            own[s] += 1
        q = query(cache, g)
        check(prefix, cache, parent, own, q, 0.125, cache.decode_attention_shared(q, 0.125))

    step()
    new = torch.empty(2, 30, 3, 64, dtype=torch.float16, device="cuda").normal_(generator=g)
    prefix.append(new, new, [20, 10], np.array([0] * 5 + [1] + [0] * 8 + [2] + [0] * 15, np.uint8))
    q = query(cache, g)
    with pytest.raises(kvc.KvcError) as e:  # a closed span that is not freed
        cache.decode_attention_shared(q, 0.125)
    assert e.value.status == 5
    prefix.compress_spans(*map(list, zip(*[(0, a, b) for a, b in prefix.pending_spans(0)])))
    step()
    prefix.evict([100, -1], [30, 1])
    step()
    parent[:] = [1, -1, 0, 1]
    cache.set_prefix(prefix, parent)
    step()
    cache.set_prefix(None)
    with pytest.raises(kvc.KvcError):
        cache.decode_attention_shared(q, 0.125)
    plain = cache.decode_attention_layers(q, 0.125)
    check(prefix, cache, [-1] * 4, own, q, 0.125, plain)


def test_equals_the_decode_of_whole_sequences_and_repeats_bit_for_bit():
    lens, parent, own = [777], [0] * 8, [1 + 5 * i for i in range(8)]
    prefix, cache, g = pair(3, 4, 80, lens, parent, own, "bf16", 80)
    q = query(cache, g)
    out = cache.decode_attention_shared(q, 0.11)
    whole = kvc.KVCache(3, 4, 80, [777 + n for n in own], "bf16", rotary_dim=80)
    blank = torch.zeros(3, sum(777 + n for n in own), 4, 80, dtype=torch.bfloat16, device="cuda")
    whole.append(blank, blank, [777 + n for n in own], np.zeros(blank.shape[1], np.uint8))
    for s, n in enumerate(own):
        for dst, src, mine in zip(rows_of(whole, s, 777 + n), rows_of(prefix, 0, 777), rows_of(cache, s, n)):
            dst.copy_(torch.cat([src, mine], 2))
    ref = whole.decode_attention_layers(q, 0.11)
    close(out, ref)
    for _ in range(3):
        assert torch.equal(cache.decode_attention_shared(q, 0.11), out)


def test_decodes_in_turn_and_on_another_stream():
    """The launches overlap where they may: results do not depend on what ran before."""
    parent, own = [0] * 8, [20] * 8
    prefix, cache, g = pair(2, 8, 64, [2000], parent, own, spare=50)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for step in range(20):
            new = torch.empty(2, 8, 8, 64, dtype=torch.float16, device="cuda").normal_(generator=g)
            cache.append(new, new, [1] * 8, [0] * 8)
            for s in range(8):
                own[s] += 1
            q = query(cache, g)
            a = cache.decode_attention_shared(q, 0.125)
            b = cache.decode_attention_layers(q, 0.125)
            c = cache.decode_attention_shared(q * 0.5, 0.25)
            if step % 5 == 4:
                side.synchronize()
                check(prefix, cache, parent, own, q, 0.125, a)
                check(prefix, cache, [-1] * 8, own, q, 0.125, b)
                assert torch.equal(a, c)


def test_refusals():
    prefix, _ = make(2, 2, 64, [10, 20])
    cache, g = make(2, 2, 64, [1, 1, 1])
    q = query(cache, g)
    with pytest.raises(kvc.KvcError) as e:
        cache.decode_attention_shared(q, 0.125)
    assert e.value.status == 5
    with pytest.raises(ValueError):
        cache.set_prefix(prefix, [0, 1])
    for parent in ([0, 1, 2], [0, -2, 1]):
        with pytest.raises(kvc.KvcError) as e:
            cache.set_prefix(prefix, parent)
        assert e.value.status == 1
    with pytest.raises(kvc.KvcError) as e:
        cache.set_prefix(cache, [0, 0, 0])
    assert e.value.status == 1
    for other in (make(1, 2, 64, [10])[0], make(2, 4, 64, [10])[0], make(2, 2, 80, [10])[0], make(2, 2, 64, [10], "bf16")[0],
                  make(2, 2, 64, [10], rot=32)[0]):
        with pytest.raises(kvc.KvcError) as e:
            cache.set_prefix(other, [0, 0, 0])
        assert e.value.status == 1
    local = kvc.KVCache(2, 2, 64, [64], policy=kvc.POLICY_LOCAL, local_ratio=0.5)
    with pytest.raises(kvc.KvcError) as e:
        cache.set_prefix(local, [0, 0, 0])
    assert e.value.status == 2
    with pytest.raises(kvc.KvcError) as e:
        kvc.kvc_set_prefix(cache.handle, prefix.handle, [0, 0, 0], torch.zeros(1024, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 1
    cache.set_prefix(prefix, [0, 1, 1])
    odd = torch.zeros(q.numel() + 1, dtype=torch.float16, device="cuda")[1:].view(q.shape)
    with pytest.raises(kvc.KvcError) as e:  # not 16-byte aligned
        cache.decode_attention_shared(odd, 0.125)
    assert e.value.status == 1
    out = torch.empty(q.shape, device="cuda")
    with pytest.raises(kvc.KvcError) as e:  # layers overlap
        kvc.kvc_decode_attention_shared(cache.handle, 0, 2, q, 64, 0.125, out, q[0].numel())
    assert e.value.status == 1
    new = torch.zeros(1, 2, 64, dtype=torch.float16, device="cuda")
    grown, _ = make(2, 2, 64, [10], spare=4)
    cache.set_prefix(grown, [0, 0, -1])
    grown.append(new, new, [1], [0], layer=0)
    with pytest.raises(kvc.KvcError) as e:  # layer 1 of the prefix is not written
        cache.decode_attention_shared(q, 0.125)
    assert e.value.status == 5
    grown.append(new, new, [1], [0], layer=1)
    cache.decode_attention_shared(q, 0.125)
    assert cache.device_status() == 0


@pytest.mark.parametrize("sizes,queries", [([33] + [8] * 16, 16), ([64] + [1] * 16, 16), ([33] + [32] * 16, 32), ([64] * 4, 64),
                                           ([64] * 8 + [8] * 8, 64), ([20] + [3] * 9, 16), ([32] * 3, 32)])
def test_groups_of_different_sizes(sizes, queries):
    """One large group does not make the others' CTAs as wide as its own; the first unit of the plan is of the first group."""
    parent = [g for g, n in enumerate(sizes) for _ in range(n)]
    own = [1 + i % 3 for i in range(len(parent))]
    lens = [130 + 7 * g for g in range(len(sizes))]
    lens[0] = 200
    prefix, cache, g = pair(1, 2, 64, lens, parent, own)
    q = query(cache, g)
    out = cache.decode_attention_shared(q, 0.125)
    check(prefix, cache, parent, own, q, 0.125, out)
    unit = cache._prefix_scratch.tensor[:32].view(torch.int32).tolist()  # prefix, rows, members' first and number, ..
    assert unit[0] == 0 and unit[4] == queries


@pytest.mark.parametrize("members", [6, 20, 40, 130])
@pytest.mark.parametrize("d,dtype,rot", [(64, "f16", 0), (64, "bf16", 64), (80, "bf16", 0), (96, "f16", 96), (128, "bf16", 128), (128, "f16", 0)])
def test_what_lies_behind_the_rows_is_not_read(members, d, dtype, rot):
    """Spare rows of K and V that hold NaN or infinities, behind prefixes whose ends lie in every part of a tile, and queries
    that are not finite: each spoils its own output only.  For every kernel and swizzle."""
    lens = [300, 129, 255, 64] if members < 130 else [300]
    parent = [g for g in range(len(lens)) for _ in range(members)]
    own = [1 + i % 3 for i in range(len(parent))]
    prefix, cache, g = pair(1, 2, d, lens, parent, own, dtype, rot, spare=70, seed=members + d)
    for c, stored in ((prefix, lens), (cache, own)):
        for plane, what in ((c.k, float("nan")), (c.v, float("inf"))):
            for s, n in enumerate(stored):
                base, cap = c.H * int(c.offsets[s]), int(c.capacity[s])
                rows = plane.view(-1, d)[base:base + 2 * cap].view(2, cap, d)
                rows[0, n:], rows[1, n:] = what, float("nan")
    q = query(cache, g)
    clean = cache.decode_attention_shared(q, d ** -0.5)
    check(prefix, cache, parent, own, q, d ** -0.5, clean)
    bad = q.clone()
    spoilt = [(2, 0), (members // 2, 1), (members - 1, 1)]
    for (s, h), what in zip(spoilt, (float("nan"), float("inf"), float("-inf"))):
        bad[0, s, h, 5] = what
    out = cache.decode_attention_shared(bad, d ** -0.5)
    for s in range(len(parent)):
        for h in range(2):
            if (s, h) in spoilt:
                assert torch.isnan(out[0, s, h]).all()
            else:
                assert torch.equal(out[0, s, h], clean[0, s, h])
    assert cache.device_status() == 0
