"""Copies of sequences and cuts on the GPU: rows, metadata, scores and what decodes afterwards."""
import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc
from _packed import CL, CR, close4, fill, held, quantise, stored, tokens, unpack16
from _serving import TDT, attend, close, collected, make, per_row, query, rows_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_fork_within_a_16_bit_cache(d, dtype):
    lens = [300, 0, 129, 0, 7, 0, 1]
    cache, g = make(2, 3, d, lens, dtype, spare=400)
    for t in (cache.k, cache.v):
        assert torch.isfinite(t).any()
    before = [[x.clone() for x in rows_of(cache, s, 300)] for s in range(7)]
    cache.copy_from(cache, [1, 3, 5, 4], [0, 0, 2, 6])
    now = [300, 300, 129, 300, 1, 129, 1]
    assert cache.lengths()[0].tolist() == now
    for s, src in ((1, 0), (3, 0), (5, 2), (4, 6), (0, 0), (2, 2), (6, 6)):
        for a, b, own in zip(rows_of(cache, s, 300), before[src], before[s]):
            n = now[s]
            assert torch.equal(a[:, :, :n], b[:, :, :n]), (s, src)
            assert torch.equal(a[:, :, n:].view(torch.int16), own[:, :, n:].view(torch.int16)), s  # what lies behind stays
        x, y = cache.masked_reference_layout(s), cache.masked_reference_layout(src)
        assert x["stored_orig"].tolist() == y["stored_orig"].tolist() == list(range(now[s]))
        assert x["stored_pos"].tolist() == y["stored_pos"].tolist()
    q = query(cache, g)
    for a, b in ((1, 0), (3, 0), (5, 2), (4, 6)):
        q[:, a] = q[:, b]
    out = cache.decode_attention_layers(q, 0.1)
    for a, b in ((1, 0), (3, 0), (5, 2), (4, 6)):
        close4(out[:, a], out[:, b])
    assert cache.device_status() == 0


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_between_16_and_4_bits(d, dtype):
    lens = [300, 5, 0, 257, 64]
    wide, g = make(2, 3, d, lens, dtype, spare=1)
    narrow = kvc.KVCache(2, 3, d, [310, 300, 9, 400, 64, 3], dtype, bits=4)
    narrow.copy_from(wide, [1, 3, 0, 4], [3, 0, 1, 4])
    assert narrow.lengths()[0].tolist() == [5, 257, 0, 300, 64, 0]
    for dst, src in ((1, 3), (3, 0), (0, 1), (4, 4)):
        n = lens[src]
        for w, x in zip("kv", rows_of(wide, src, n)):
            for a, b in zip(stored(narrow, dst, n, w), quantise(x)):
                assert torch.equal(a, b), (dst, w)
    # within 4 bits, an odd number of rows among them
    narrow.copy_from(narrow, [0], [1])
    for w in "kv":
        for a, b in zip(stored(narrow, 0, 257, w), stored(narrow, 1, 257, w)):
            assert torch.equal(a, b)
    # and back: the values that the codes stand for, rounded once
    back = unpack16(narrow)
    for s, src in ((0, 3), (1, 3), (3, 0), (4, 4)):
        n = lens[src]
        for a, x in zip(rows_of(back, s, n), rows_of(wide, src, n)):
            assert torch.equal(a.cpu(), held(x.contiguous()).cpu().float().to(TDT[dtype])), s
    lay = back.masked_reference_layout(3)
    assert lay["stored_orig"].tolist() == list(range(300))
    # a decode over the 4 bits is one over the values
    q = query(narrow, g)
    out = narrow.decode_attention_layers(q, 0.1)
    if dtype == "f16":
        assert float((out[:, 3] - back.decode_attention_layers(q, 0.1)[:, 3]).norm() / out[:, 3].norm()) < 2e-3


@pytest.mark.parametrize("bits", [(16, 16), (16, 4), (4, 4), (4, 16)])
def test_uneven_sources_and_empty_ones(bits):
    """Runs of rows that end with a source's last row, at a block's edge and one to either side of it; sources without rows
    among the others free their targets."""
    lens = [0, 1500, 0, 1, 127, 128, 129, 255, 256, 257, 0, 513]
    b = len(lens)
    a, g, k, v = fill(2, 2, 80, lens, "bf16", bits=bits[0])
    c, _, _, _ = fill(2, 2, 80, [3] * (2 * b), "bf16", spare=1600, bits=bits[1], seed=5)
    order = [int(x) for x in np.random.default_rng(3).permutation(2 * b)]
    src = [i % b for i in range(2 * b)]
    c.copy_from(a, order, src)
    assert [c.lengths()[0][d] for d in order] == [lens[s] for s in src]
    for d, s in zip(order, src):
        if lens[s] == 0:
            continue
        for w, x in zip("kv", (k, v)):
            rows = tokens(x, lens, s)
            if bits[1] == 4:
                for got, want in zip(stored(c, d, lens[s], w), quantise(rows)):
                    assert torch.equal(got, want), (d, s, w)
            else:
                want = rows if bits[0] == 16 else held(rows).float().to(rows.dtype)
                assert torch.equal(rows_of(c, d, lens[s])["kv".index(w)], want), (d, s, w)
        assert c.masked_reference_layout(d)["stored_pos"].tolist() == list(range(lens[s]))
    assert c.device_status() == 0


def test_rows_behind_the_last_stay():
    narrow, g, _, _ = fill(1, 2, 80, [40, 13, 0], "f16", spare=30)
    for t in (narrow.k, narrow.v):
        t.random_(0, 256, generator=g)
    k0, v0 = narrow.k.clone(), narrow.v.clone()
    narrow.copy_from(narrow, [2], [1])
    for before, after in ((k0, narrow.k), (v0, narrow.v)):
        changed = (before != after).nonzero().flatten().tolist()
        rows = 2 * narrow.C
        code = [i // 40 for i in changed if i < rows * 40]
        start = (rows * 40 + 255) // 256 * 256
        pair = [(i - start) // 12 for i in changed if i >= start]
        base = 2 * int(narrow.offsets[2])  # capacity 31, 32 rows in the layout
        allowed = set(range(base, base + 13)) | set(range(base + 32, base + 45))
        assert set(code) <= allowed and set(pair) <= allowed and code and pair


def test_many_copies_at_once():
    """More sequences than the kernel parameter holds."""
    b = 300
    lens = [3 + i % 7 for i in range(b // 2)] + [0] * (b // 2)
    for bits in (16, 4):
        cache, g, k, v = fill(1, 2, 64, lens, "f16", spare=10, bits=bits)
        cache.copy_from(cache, range(b // 2, b), range(b // 2))
        q = query(cache, g)
        q[:, b // 2:] = q[:, :b // 2]
        out = cache.decode_attention_layers(q, 0.1)
        close4(out[:, b // 2:], out[:, :b // 2])
        cache.truncate([i % 4 for i in range(b)])
        assert cache.lengths()[0].tolist() == [i % 4 for i in range(b)]
        short = cache.decode_attention_layers(q, 0.1, out=torch.zeros_like(out))
        plain, _, _, _ = fill(1, 2, 64, lens, "f16", spare=10, bits=bits)
        plain.truncate([i % 4 for i in range(b // 2)] + [-1] * (b // 2))
        want = plain.decode_attention_layers(q, 0.1, out=torch.zeros_like(out))
        close4(short[:, :b // 2], want[:, :b // 2])
        assert cache.device_status() == 0


def test_spans_and_evictions_go_along():
    lens = [200, 120, 0, 0]
    kinds = [np.zeros(n, np.uint8) for n in lens]
    kinds[0][50], kinds[0][90] = CL, CR
    kinds[0][150] = CL
    cache, g = make(2, 2, 64, lens, spare=200, kinds=kinds)
    scores = cache.attach_scores()
    for s in (0, 1):
        per_row(cache, scores, s, lens[s]).uniform_(0.5, 1.0, generator=g)
    cache.evict([-1, 60, -1, -1], [1, 20, 1, 1])
    cache.copy_from(cache, [2, 3], [0, 1])
    for s, src, n in ((2, 0, 200), (3, 1, 60)):
        assert torch.equal(per_row(cache, scores, s, n), per_row(cache, scores, src, n))
    q = query(cache, g)
    q[:, 2:] = q[:, :2]
    assert cache.pending_spans(2) == [(50, 90)]
    cache.compress_spans([0, 2], [50, 50], [90, 90])
    out = cache.decode_attention_layers(q, 0.1)  # the open span's <CL> is as hidden in the copy
    close4(out[:, 2:], out[:, :2])
    # an evicted copy is evicted on
    cache.evict([-1, 30, -1, 30], [1, 10, 1, 10])
    for a, b in zip(rows_of(cache, 1, 30), rows_of(cache, 3, 30)):
        assert torch.equal(a, b)
    # scores where the source's cache has none: 0, and none left of the rows that were there
    other, _ = make(2, 2, 64, [10], seed=4)
    cache.copy_from(other, [1], [0])
    cap = int(cache.capacity[1])
    assert (per_row(cache, scores, 1, cap) == 0).all()
    # and slots without a row hold 0 after a cut
    cache.truncate([20, -1, -1, 0])
    assert (per_row(cache, scores, 0, 400)[:, :, 20:] == 0).all() and (per_row(cache, scores, 0, 20) > 0).all()
    assert (per_row(cache, scores, 3, 200) == 0).all()
    assert (per_row(cache, scores, 2, 5) > 0).all()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("d", [64, 80])
def test_cut_and_go_on(bits, d):
    """Drafted tokens that are dropped leave no trace: the cache goes on like one that never had them."""
    lens = [70, 5]
    a, g, k, v = fill(2, 2, d, lens, "f16", spare=60, bits=bits, rot=16)
    b, _, _, _ = fill(2, 2, d, lens, "f16", spare=60, bits=bits, rot=16)
    q = query(a, g)
    draft = [torch.randn(2, 11, 2, d, device="cuda").half() for _ in range(2)]
    a.append(*draft, [9, 2], np.array([0, CL, 0, CR, 0, 0, CL, 0, 0, 0, 0], np.uint8))
    a.truncate([70, 6])
    b.append(draft[0][:, 9:10].contiguous(), draft[1][:, 9:10].contiguous(), [0, 1], np.zeros(1, np.uint8))
    assert torch.equal(a.decode_attention_layers(q, 0.1), b.decode_attention_layers(q, 0.1))
    more = [torch.randn(2, 8, 2, d, device="cuda").half() for _ in range(2)]
    for c in (a, b):
        c.append(*more, [5, 3], np.zeros(8, np.uint8))
    assert torch.equal(a.decode_attention_layers(q, 0.1), b.decode_attention_layers(q, 0.1))
    # a freed sequence begins anew
    for c in (a, b):
        c.truncate([0, -1])
    out = torch.full((2, 2, 2, d), 3.0, device="cuda")
    a.decode_attention_layers(q, 0.1, out=out)
    assert (out[:, 0] == 3.0).all()
    a.append(*[x[:, :4].contiguous() for x in draft], [4, 0], np.zeros(4, np.uint8))
    assert a.masked_reference_layout(0)["stored_pos"].tolist() == [0, 1, 2, 3]
    one, _, _, _ = fill(2, 2, d, [0, 0], "f16", spare=60, bits=bits, rot=16)
    one.append(*[x[:, :4].contiguous() for x in draft], [4, 0], np.zeros(4, np.uint8))
    close4(a.decode_attention_layers(q, 0.1)[:, 0], one.decode_attention_layers(q, 0.1, out=torch.zeros_like(out))[:, 0])
    assert a.device_status() == 0


def test_a_prompt_in_16_bits_and_its_samples_in_4():
    """As they are used together: a prompt's prefill and compaction in 16 bits, samples forked into a 4-bit cache, steps there,
    beams that replace others, drafts that go, and a session that comes back for its next prompt."""
    M, H, d = 2, 4, 64
    n, kinds = 200, np.zeros(200, np.uint8)
    kinds[40], kinds[120] = CL, CR
    prompt, g = make(M, H, d, [n], spare=300, kinds=[kinds])
    for m in range(M):
        prompt.prefill_attention(m, torch.randn(n, H, d, device="cuda").half(), [n], 0.1)
    prompt.compress_spans([0], [40], [120])
    cache = kvc.KVCache(M, H, d, [400] * 4, "f16", bits=4)
    cache.copy_from(prompt, [0, 1, 2, 3], [0] * 4)
    keep = n - 80
    record = [rows_of(prompt, 0, keep)[0].clone(), rows_of(prompt, 0, keep)[1].clone()]
    rows = [[x for x in record] for _ in range(4)]
    for step in range(6):
        new = [torch.randn(M, 4, H, d, device="cuda").half() for _ in range(2)]
        cache.append(*new, [1] * 4, np.zeros(4, np.uint8))
        for s in range(4):
            rows[s] = [torch.cat([r, x[:, s, :, None]], 2) for r, x in zip(rows[s], new)]
        if step == 2:  # sample 0 goes on in place of sample 3
            cache.copy_from(cache, [3], [0])
            rows[3] = list(rows[0])
        if step == 4:  # sample 1's last two tokens were drafts
            cache.truncate([-1, n + step - 1, -1, -1])
            rows[1] = [r[:, :, :-2] for r in rows[1]]
        q = query(cache, g)
        out = cache.decode_attention_layers(q, 0.1)
        for s in range(4):
            k, v = (held(r.contiguous()) for r in rows[s])
            w = torch.softmax(torch.einsum("mhd,mhnd->mhn", q[:, s].double(), k) * 0.1, -1)
            close4(out[:, s], torch.einsum("mhn,mhnd->mhd", w, v), f"step {step} sample {s}")
    # the session comes back
    prompt.copy_from(cache, [0], [2])
    got = rows_of(prompt, 0, keep + 6)
    for a, r in zip(got, rows[2]):
        assert torch.equal(a, held(r.contiguous()).float().half())
    block = [torch.randn(M, 30, H, d, device="cuda").half() for _ in range(2)]
    prompt.append(*block, [30], np.zeros(30, np.uint8))
    prompt.prefill_attention(0, torch.randn(30, H, d, device="cuda").half(), [30], 0.1)
    for c in (prompt, cache):
        assert c.device_status() == 0


def test_streams_and_graphs():
    cache, g, _, _ = fill(2, 2, 64, [50, 0, 0], "f16", spare=60, bits=4)
    wide, _ = make(2, 2, 64, [50, 20], seed=2, spare=60)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache.copy_from(wide, [1, 2], [0, 1], stream=side)
    side.synchronize()
    assert cache.lengths()[0].tolist() == [50, 50, 20]
    ref = [stored(cache, s, n) for s, n in ((1, 50), (2, 20))]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.copy_from(wide, [1, 2], [0, 1])
    cache.k.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for (s, n), r in zip(((1, 50), (2, 20)), ref):
        for a, b in zip(stored(cache, s, n), r):
            assert torch.equal(a, b)
    # of more sequences than a parameter holds: refused in a capture, nothing changed
    many, _, _, _ = fill(1, 1, 64, [2] * 200, "f16", spare=2, bits=4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in (lambda: many.truncate(1), lambda: many.copy_from(many, [0], [1])):
            with pytest.raises(kvc.KvcError) as e:
                call()
            assert e.value.status == 5
    assert many.lengths()[0].tolist() == [2] * 200
    many.truncate(1)


@pytest.mark.parametrize("d", [64, 128])
def test_prefixes_copied_and_cut(d):
    """Copies and cuts of a shared prefix and of the sequences over it: each decode is over the rows that are there then."""
    prefix, _ = make(2, 3, d, [300, 40], spare=300)
    parent, own = [0, 0, 1, -1], [3, 1, 2, 5]
    pos = np.concatenate([(0 if p < 0 else 40) + np.arange(n) for p, n in zip(parent, own)]).astype(np.int32)
    cache, g = make(2, 3, d, own, seed=1, spare=9, pos=pos)
    cache.set_prefix(prefix, parent)

    def check(plen, own):
        q = query(cache, g)
        out = cache.decode_attention_shared(q, 0.1)
        assert prefix.lengths()[0].tolist() == plen and cache.lengths()[0].tolist() == own
        for s, (p, n) in enumerate(zip(parent, own)):
            k, v = rows_of(cache, s, n)
            if p >= 0:
                k, v = (torch.cat(x, 2) for x in zip(rows_of(prefix, p, plen[p]), (k, v)))
            for m in range(2):
                close(out[m, s], attend(q[m, s].double(), k[m], v[m], list(range(k.shape[2])), 0.1)[0], f"sequence {s}")

    check([300, 40], own)
    prefix.truncate([130, -1])
    check([130, 40], own)
    prefix.copy_from(prefix, [1], [0])
    check([130, 130], own)
    other, _ = make(2, 3, d, [257, 3], seed=2)
    prefix.copy_from(other, [0, 1], [1, 0])
    check([3, 257], own)
    cache.copy_from(cache, [2, 3], [0, 1])  # own rows alone: sequence 2 stays over prefix 1, sequence 3 over none
    check([3, 257], [3, 1, 3, 1])
    cache.truncate([1, -1, 2, -1])
    check([3, 257], [1, 1, 2, 1])
    prefix.truncate([0, -1])
    check([0, 257], [1, 1, 2, 1])
    for c in (prefix, cache):
        assert c.device_status() == 0


def test_prompts_after_copies_and_cuts():
    """A block's attention and scores are over the rows that are there, though an earlier call had as many queries."""
    lens, n_q = [200, 90, 30], [20, 7, 11]
    a, g = make(2, 4, 64, lens, spare=200)
    k, v = (torch.empty(2, 38, 4, 64, device="cuda", dtype=torch.float16).normal_(generator=g) for _ in range(2))
    q = torch.empty(38, 4, 64, device="cuda", dtype=torch.float16).normal_(0.0, 2.0, generator=g)
    scores = a.attach_scores()

    def block():
        a.append(k, v, n_q, np.zeros(38, np.uint8))
        out = a.prefill_attention(0, q, n_q, 0.1)
        scores.zero_()
        a.score_prompt(0, q, n_q, 0.1)
        return out

    def check(out, before):
        t = 0
        for s, (n, m) in enumerate(zip(before, n_q)):
            rows = [x[0] for x in rows_of(a, s, n + m)]
            total = torch.zeros(4, n + m, dtype=torch.float64, device="cuda")
            for i in range(m):
                ref, w = attend(q[t + i].double(), *rows, list(range(n + i + 1)), 0.1)
                # a weight that the tensor cores take is rounded to 16 bits: by 2^-11 = 4.9e-4 of itself at most, and so at
                # most are the outputs and their sums; the logits in 32 bits add 1.2e-4
                assert float((out[t + i].double() - ref).norm() / ref.norm()) < 2e-3
                total[:, :n + i + 1] += w
            got = per_row(a, scores, s, n + m)[0].double()
            assert float((got - total).norm() / total.norm()) < 2e-3
            t += m

    check(block(), lens)
    a.truncate([150, 90, 0])
    check(block(), [150, 90, 0])
    a.copy_from(a, [0], [1])
    check(block(), [97, 97, 11])
    a.copy_from(a, [2], [0])
    a.truncate([3, -1, 60])
    check(block(), [3, 104, 60])
    assert a.device_status() == 0


def test_refusals_leave_the_cache():
    cache, g, _, _ = fill(2, 2, 64, [50, 9], "f16", spare=4, bits=4)
    before = (cache.k.clone(), cache.v.clone())
    wide, _ = make(2, 2, 64, [50])
    closed, _ = make(2, 2, 64, [5])
    closed.close()
    one = torch.randn(2, 2, 64, device="cuda").half()
    pending, _ = make(2, 2, 64, [5], spare=4)
    pending.append(one[:1].contiguous(), one[:1].contiguous(), [1], np.zeros(1, np.uint8), layer=0)
    for call, status in ((lambda: cache.copy_from(wide, [1], [0]), 3), (lambda: cache.copy_from(closed, [1], [0]), 5),
                         (lambda: cache.copy_from(pending, [1], [0]), 5), (lambda: pending.truncate(2), 5),
                         (lambda: cache.copy_from(cache, [1], [1]), 1), (lambda: cache.truncate([51, 0]), 1)):
        with pytest.raises(kvc.KvcError) as e:
            call()
        assert e.value.status == status
    with pytest.raises(ValueError):
        cache.truncate([1, 2, 3])
    assert cache.lengths()[0].tolist() == [50, 9]
    assert torch.equal(cache.k, before[0]) and torch.equal(cache.v, before[1])
