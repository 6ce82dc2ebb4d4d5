"""A cache of 4 bits on the GPU: what an append stores, and the decode over it, against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc
from _packed import CL, CR, N, close4, fill, held, quantise, stored, tokens, values
from _serving import TDT, attend, collected, query, rotate  # noqa: F401

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------------------------
# Append
# --------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("H", [1, 3])
def test_append_stores_the_defined_codes(d, dtype, H):
    lens = [1, 9, 0, 70]
    cache, g, k, v = fill(2, H, d, lens, dtype, spare=3)
    # then a token each (the upload as a kernel parameter), and a layer at a time
    step = [torch.empty(2, 3, H, d, dtype=TDT[dtype], device="cuda").normal_(0, 30, generator=g) for _ in range(2)]
    cache.append(*step, [1, 1, 0, 1], np.zeros(3, np.uint8))
    last = [torch.empty(2, 2, H, d, dtype=TDT[dtype], device="cuda").normal_(0, 1e-3, generator=g) for _ in range(2)]
    for m in range(2):
        cache.append(last[0][m].contiguous(), last[1][m].contiguous(), [0, 1, 1, 0], np.zeros(2, np.uint8), layer=m)
    at1, at2 = [0, 1, None, 2], [None, 0, 1, None]
    for which, x in (("k", 0), ("v", 1)):
        for s, n in enumerate(lens):
            rows = [tokens((k, v)[x], lens, s)]
            if at1[s] is not None:
                rows.append(step[x][:, at1[s], :, None])
            if at2[s] is not None:
                rows.append(last[x][:, at2[s], :, None])
            rows = torch.cat(rows, 2)
            got = stored(cache, s, rows.shape[2], which)
            for a, b, name in zip(got, quantise(rows), ("codes", "steps", "least values")):
                assert torch.equal(a, b), (which, s, name)
    assert cache.device_status() == 0


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_append_of_unusual_rows(dtype):
    d, big = 80, 65504.0 if dtype == "f16" else 1e38
    tiny = 2.0 ** -24 if dtype == "f16" else 2.0 ** -133
    rows = torch.zeros(8, d)
    rows[1] = 3.0
    rows[2, ::2], rows[2, 1::2] = big, -big
    rows[3] = torch.arange(d) * tiny
    rows[4] = -torch.arange(d) * tiny * 7
    rows[5, 40] = 1.0
    rows[6] = torch.linspace(-1e-3, 1e-3, d)
    rows[7] = torch.arange(d) % 16  # on the levels
    x = rows.to(TDT[dtype]).cuda()[None, :, None].contiguous()
    cache = kvc.KVCache(1, 1, d, [8], dtype, bits=4)
    cache.append(x, x, [8], np.zeros(8, np.uint8))
    want = quantise(x[0, :, 0])
    for which in "kv":
        got = stored(cache, 0, 8, which)
        for a, b, name in zip(got, want, ("codes", "steps", "least values")):
            assert torch.equal(a[0, 0], b), (which, name)
    err = (values(*want) - x[0, :, 0].double().cpu()).abs()
    # a step is 0 only where a fifteenth of the range is below 2^-126: every column is then within 15 x 2^-126 of the least one
    allowed = torch.where(want[1] > 0, want[1] * 0.5 * (1 + 2.0 ** -20), 15 * 2.0 ** -126)
    for g, a in enumerate(range(0, d, 32)):
        assert (err[:, a:a + 32] <= allowed[:, g:g + 1]).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_groups_that_are_not_finite_read_as_nan_alone(dtype):
    d = 96
    x = torch.randn(5, d).to(TDT[dtype])
    x[1, 3], x[2, 40], x[3, 95] = math.nan, math.inf, -math.inf
    ref = held(torch.where(torch.isfinite(x), x, torch.zeros_like(x)))
    x = x.cuda()[None, :, None].contiguous()
    cache = kvc.KVCache(1, 1, d, [5], dtype, bits=4)
    cache.append(x, x, [5], np.zeros(5, np.uint8))
    got = values(*stored(cache, 0, 5))[0, 0]
    bad = torch.zeros(5, d, dtype=torch.bool)
    bad[1, :32] = bad[2, 32:64] = bad[3, 64:] = True
    assert torch.isnan(got[bad]).all()
    assert torch.equal(got[~bad], ref[~bad])


@pytest.mark.parametrize("d,rot", [(64, 64), (80, 48), (96, 16), (128, 128)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_rotated_keys(d, rot, dtype):
    """The codes are those of the keys that a 16-bit cache holds, up to that cache's own rounding of a rotated key."""
    lens = [37, 5]
    cache, _, k, v = fill(2, 3, d, lens, dtype, rot=rot, spare=2)
    wide = kvc.KVCache(2, 3, d, [40, 8], dtype, rotary_dim=rot)
    wide.append(k, v, lens, np.zeros(42, np.uint8))
    one = [x[:, :2].contiguous() for x in (k, v)]
    for c in (cache, wide):
        c.append(*one, [1, 1], np.zeros(2, np.uint8))
    eps = torch.finfo(TDT[dtype]).eps
    for s, n in enumerate(lens):
        codes, step, lo = stored(cache, s, n + 1)
        got = values(codes, step, lo)
        for m in range(2):
            for h in range(3):
                x = wide.stream_rows(wide.k_plane(m), s, h, n + 1).cpu().double()
                for g, a in enumerate(range(0, d, 32)):
                    part = x[:, a:a + 32]
                    # half a step, and a key that was rounded to the neighbouring value (also as the group's least or
                    # greatest, from which the step follows)
                    allowed = step[m, h][:, g:g + 1] * 0.5 * (1 + 2.0 ** -20) + 2 * eps * part.abs().amax(-1, keepdim=True)
                    assert ((got[m, h][:, a:a + 32] - part).abs() <= allowed).all()


# --------------------------------------------------------------------------------------------
# Decode
# --------------------------------------------------------------------------------------------

def reference(cache, s, q, n, rows, scale, pos):
    """out [M, H, d] of sequence s over the given rows of what it holds."""
    k, v = (values(*stored(cache, s, n, w)) for w in "kv")
    return torch.stack([attend(rotate(q[m, s].cpu(), pos, cache.rotary_dim), k[m], v[m], rows, scale)[0] for m in range(cache.M)])


def check(cache, q, lens, scale, out=None, what=""):
    got = cache.decode_attention_layers(q, scale, out=out)
    for s, n in enumerate(lens):
        if n:
            lay = cache.book.layout(s)
            ref = reference(cache, s, q, n, range(n), scale, int(lay["pos"][-1]))
            close4(got[:, s], ref, f"{what} sequence {s} of {n} rows")
    return got


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rotated", [0, 1])
def test_decode_of_all_lengths(d, dtype, rotated):
    lens = [1, 2, 3, 4, 5, 0, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257, 511]
    cache, g, _, _ = fill(2, 3, d, lens, dtype, rot=rotated * 48, spare=1)
    q = query(cache, g)
    out = torch.full((2, len(lens), 3, d), 7.0, device="cuda")
    check(cache, q, lens, 1 / math.sqrt(d), out)
    assert (out[:, 5] == 7.0).all()  # no token: left as it was
    assert cache.device_status() == 0
    # each layer by itself
    for m in range(2):
        one = cache.decode_attention(m, q[m].contiguous(), 1 / math.sqrt(d), out=out[m].clone())
        close4(one, out[m], "one layer")


@pytest.mark.parametrize("M,H,lens", [(1, 1, [1]), (1, 1, [70001]), (3, 5, [9000, 40, 1]), (1, 2, [300] * 70), (24, 8, [200, 130]),
                                      (2, 40, [1000, 3, 700])])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (80, "f16"), (128, "f16")])
def test_decode_of_few_and_many_segments(M, H, lens, d, dtype):
    cache, g, _, _ = fill(M, H, d, lens, dtype, seed=3)
    q = query(cache, g)
    first = check(cache, q, lens, 0.1)
    for _ in range(3):  # one order of additions
        assert torch.equal(cache.decode_attention_layers(q, 0.1), first)
    assert cache.device_status() == 0


@pytest.mark.parametrize("policy", [kvc.POLICY_PAPER, kvc.POLICY_KEEP_CL])
@pytest.mark.parametrize("d", [64, 96])
def test_decode_masks_and_compaction(policy, d):
    """An open span's <CL>, a <CL> query, a closed span that is not freed, and the rows that are left once it is."""
    lens = [150, 66, 40, 300]
    kinds = [np.zeros(n, np.uint8) for n in lens]
    kinds[0][100] = CL                       # open
    kinds[1][65] = CL                        # the query
    kinds[2][5], kinds[2][39] = CL, CR       # closed by the query
    kinds[3][70], kinds[3][140] = CL, CR     # closed before it
    cache, g, k, v = fill(2, 2, d, lens, "f16", kinds=kinds, policy=policy, spare=4)
    paper = policy == kvc.POLICY_PAPER
    rows = [[i for i in range(150) if not (paper and i == 100)], [65], [i for i in range(40) if not (paper and i == 5)],
            [i for i in range(300) if not (70 + (not paper) <= i < 140)]]
    q = query(cache, g)
    got = cache.decode_attention_layers(q, 0.125)
    for s, n in enumerate(lens):
        close4(got[:, s], reference(cache, s, q, n, rows[s], 0.125, 0), f"sequence {s}")
    before = [stored(cache, s, n, w) for s, n in enumerate(lens) for w in "kv"]
    cache.compress_spans([3, 2], [70, 5], [140, 39])
    rows[2] = [i for i in range(40) if not (5 + (not paper) <= i < 39)]
    assert cache.lengths()[0].tolist() == [150, 66, len(rows[2]), len(rows[3])]
    for s in range(4):
        kept = rows[s] if s >= 2 else list(range(lens[s]))
        for w in range(2):
            now = stored(cache, s, len(kept), "kv"[w])
            for a, b in zip(now, before[2 * s + w]):
                assert torch.equal(a, b[:, :, kept])
    lay = cache.masked_reference_layout(3)
    assert lay["stored_orig"].tolist() == rows[3]
    again = cache.decode_attention_layers(q, 0.125)
    close4(again[:, 3], got[:, 3], "freed")
    # the sequences go on: appended rows follow the ones that are left
    new = [torch.randn(2, 4, 2, d, device="cuda").half() for _ in range(2)]
    cache.append(*new, [1, 1, 1, 1], np.array([N] * 4, np.uint8))
    out = cache.decode_attention_layers(q, 0.125)
    n = len(rows[3]) + 1
    close4(out[:, 3], reference(cache, 3, q, n, range(n), 0.125, 0), "appended")
    assert torch.equal(stored(cache, 3, n)[0][:, :, -1], quantise(new[0][:, 3])[0])


@pytest.mark.parametrize("d", [64, 80, 128])
def test_compaction_of_many_spans(d):
    n, kinds = 700, np.zeros(700, np.uint8)
    spans = [(a, a + 9) for a in range(3, 680, 17)]
    for a, z in spans:
        kinds[a], kinds[z] = CL, CR
    cache, g, _, _ = fill(3, 2, d, [n], "bf16", kinds=[kinds])
    before = [stored(cache, 0, n, w) for w in "kv"]
    cache.compress_spans([0] * len(spans), *zip(*spans))
    kept = [i for i in range(n) if not any(a <= i < z for a, z in spans)]
    for w in range(2):
        for a, b in zip(stored(cache, 0, len(kept), "kv"[w]), before[w]):
            assert torch.equal(a, b[:, :, kept])
    assert cache.device_status() == 0


def test_freed_as_it_is_written():
    kinds = np.zeros(60, np.uint8)
    kinds[10], kinds[30] = CL, CR
    cache = kvc.KVCache(1, 2, 64, [64], "f16", bits=4)
    x = torch.randn(1, 60, 2, 64, device="cuda").half()
    cache.append(x, x, [60], kinds, free_closed=True)
    kept = [i for i in range(60) if not 10 <= i < 30]
    for a, b in zip(stored(cache, 0, 40), quantise(x[:, kept].transpose(1, 2))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_values_of_every_size(d, dtype):
    """Rows and queries far from 1: the parts that go into the products do not run over or vanish."""
    sizes = [1e-6, 1e-3, 1.0, 300.0] + ([1e-25, 1e25] if dtype == "bf16" else [])
    for kv in sizes:
        for sq in [1e-4, 1.0, 1e4] + ([1e-11, 1e11] if dtype == "bf16" else []):
            g = torch.Generator(device="cuda")
            g.manual_seed(7)
            cache = kvc.KVCache(1, 2, d, [300], dtype, bits=4)
            k, v = (torch.empty(1, 300, 2, d, device="cuda").normal_(generator=g) * kv for _ in range(2))
            cache.append(k.to(TDT[dtype]), v.to(TDT[dtype]), [300], np.zeros(300, np.uint8))
            q = (torch.empty(1, 1, 2, d, device="cuda").normal_(generator=g) * sq).to(TDT[dtype])
            scale = 0.1 / (kv * sq)
            check(cache, q, [300], scale, what=f"rows {kv} query {sq}")
    # columns of very different sizes, and rows too
    cache = kvc.KVCache(1, 2, d, [300], dtype, bits=4)
    k = torch.randn(1, 300, 2, d, device="cuda")
    v = k * (10.0 ** torch.linspace(-4, 2, 300, device="cuda"))[None, :, None, None]
    k[..., 5] *= 50
    cache.append(k.to(TDT[dtype]), v.to(TDT[dtype]), [300], np.zeros(300, np.uint8))
    q = torch.randn(1, 1, 2, d, device="cuda").to(TDT[dtype])
    check(cache, q, [300], 0.05)


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_values_that_are_not_finite(d, dtype):
    """A query that is not finite gets NaN; a NaN among the keys' groups makes its logit NaN; among the values its columns;
    none reaches a query that does not see the row."""
    lens = [100, 100, 100, 100, 100]
    kinds = [np.zeros(n, np.uint8) for n in lens]
    kinds[4][60] = CL
    cache = kvc.KVCache(1, 2, d, [100] * 5, dtype, bits=4)
    k, v = (torch.randn(1, 500, 2, d, device="cuda").to(TDT[dtype]) for _ in range(2))
    k[:, 150, 0, 3] = math.nan
    v[:, 250, 1, 40] = -math.inf
    k[:, 460], v[:, 460] = math.nan, math.inf  # the hidden <CL> row
    cache.append(k, v, lens, np.concatenate(kinds))
    q = torch.randn(1, 5, 2, d, device="cuda").to(TDT[dtype])
    q[0, 3, 0, 7] = math.inf
    out = cache.decode_attention_layers(q, 0.125)[0]
    nan = torch.isnan(out).cpu()
    want = torch.zeros_like(nan)
    want[1, 0] = want[3, 0] = True
    want[2, 1, 32:64] = True
    assert torch.equal(nan, want)
    k2, v2 = (values(*stored(cache, 2, 100, w))[0, 1:] for w in "kv")  # the other columns beside those that are NaN
    rest = [c for c in range(d) if not 32 <= c < 64]
    close4(out[2, 1:, rest], attend(q[0, 2, 1:].double().cpu(), k2, v2, range(100), 0.125)[0][:, rest], "beside")
    rows = [i for i in range(100) if i != 60]
    close4(out[4], reference(cache, 4, q, 100, rows, 0.125, 0)[0], "hidden row")
    close4(out[0], reference(cache, 0, q, 100, range(100), 0.125, 0)[0], "plain")


def test_offsets_past_32_bits():
    M, H, d, cap = 40, 40, 128, 40000
    cache = kvc.KVCache(M, H, d, [cap, cap], "f16", bits=4)  # 1.28e8 rows, 8.2 GB of codes a side
    x = torch.randn(1, 5 + 70, H, d, device="cuda").half().expand(M, -1, -1, -1).contiguous()
    cache.append(x, x, [5, 70], np.zeros(75, np.uint8))
    q = torch.randn(1, 2, H, d, device="cuda").half().expand(M, -1, -1, -1).contiguous()
    out = cache.decode_attention_layers(q, 0.1)
    for m in range(M):  # not bit for bit: the workers' shares end elsewhere in each layer's segments
        close4(out[m], out[0], f"layer {m}")
    small = kvc.KVCache(1, H, d, [8, 80], "f16", bits=4)
    small.append(x[:1].contiguous(), x[:1].contiguous(), [5, 70], np.zeros(75, np.uint8))
    close4(out[:1], small.decode_attention_layers(q[:1].contiguous(), 0.1), "small")
    assert cache.device_status() == 0


def test_strides_streams_and_graphs():
    cache, g, _, _ = fill(3, 2, 64, [500, 77], "f16", spare=9)
    q = query(cache, g)
    ref = cache.decode_attention_layers(q, 0.1)
    # layers apart by more than a layer, and queries at an odd element
    n = 2 * 2 * 64
    qs = torch.zeros(1 + 3 * (n + 13), dtype=torch.float16, device="cuda")
    outs = torch.full((3 * (n + 7),), 5.0, device="cuda")
    for m in range(3):
        qs[1 + m * (n + 13):1 + m * (n + 13) + n] = q[m].flatten()
    kvc.kvc_decode_attention_layers(cache.handle, 0, 3, qs[1:], n + 13, 0.1, outs, n + 7)
    for m in range(3):
        assert torch.equal(outs[m * (n + 7):m * (n + 7) + n], ref[m].flatten())
        assert (outs[m * (n + 7) + n:(m + 1) * (n + 7)] == 5.0).all()
    # another stream, back to back calls
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = [torch.empty_like(ref) for _ in range(6)]
    for o in out:
        cache.decode_attention_layers(q, 0.1, out=o, stream=side)
    side.synchronize()
    assert all(torch.equal(o, ref) for o in out)
    # a graph, replayed with other queries
    graph, o = torch.cuda.CUDAGraph(), torch.empty_like(ref)
    with torch.cuda.graph(graph):
        for _ in range(3):
            cache.decode_attention_layers(q, 0.1, out=o)
    q2 = query(cache, g)
    q.copy_(q2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, cache.decode_attention_layers(q2, 0.1))
    # a step and its decode, many times: each sees the row before it
    for i in range(8):
        x = torch.randn(3, 2, 2, 64, device="cuda").half()
        cache.append(x, x, [1, 1], np.zeros(2, np.uint8))
        got = cache.decode_attention_layers(q2, 0.1)
        if i in (0, 7):
            close4(got[:, 1], reference(cache, 1, q2, 78 + i, range(78 + i), 0.1, 0), f"step {i}")
    assert cache.device_status() == 0


def test_refusals_of_a_live_cache():
    cache, g, _, _ = fill(1, 2, 64, [10], "f16")
    q = query(cache, g)
    out = torch.empty(1, 2, 64, device="cuda")
    calls = [lambda: kvc.kvc_decode_attention_static_scratch(cache.handle, 0, q, 0.1, out),
             lambda: cache.prefill_attention(0, q[0], [1], 0.1), lambda: cache.attach_scores(),
             lambda: cache.decode_attention_shared(q, 0.1), lambda: cache.evict(5, 2), lambda: cache.k_plane(0)]
    for i, call in enumerate(calls):
        with pytest.raises(kvc.KvcError) as e:
            call()
        assert e.value.status == (5 if i == 3 else 2), i
    with pytest.raises(kvc.KvcError) as e:
        cache.decode_attention_scored(q, 0.1)
    assert e.value.status == 5  # no scores
    cache.decode_attention_layers(q, 0.1)


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (80, "bf16"), (128, "f16")])
def test_hidden_runs_over_whole_tiles_and_workers(d, dtype):
    """Parts without a visible row: a span that is closed and not freed covers whole tiles, and the shares of whole workers."""
    lens = [300, 20011, 130]
    kinds = [np.zeros(n, np.uint8) for n in lens]
    kinds[0][1], kinds[0][290] = CL, CR
    kinds[1][0], kinds[1][20009] = CL, CR
    kinds[2][3], kinds[2][128] = CL, CR
    cache, g, _, _ = fill(1, 2, d, lens, dtype, kinds=kinds)
    q = query(cache, g)
    got = cache.decode_attention_layers(q, 0.1)
    for s, (n, a, z) in enumerate(zip(lens, (1, 0, 3), (290, 20009, 128))):
        rows = [i for i in range(n) if not a <= i < z]
        close4(got[:, s], reference(cache, s, q, n, rows, 0.1, 0), f"sequence {s}")
    cache.compress_spans([0, 1, 2], [1, 0, 3], [290, 20009, 128])
    again = cache.decode_attention_layers(q, 0.1)
    close4(again, got, "freed")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 96])
def test_queries_scales_and_rows_at_the_edge(d, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    k, v = (torch.empty(1, 200, 2, d, device="cuda").normal_(generator=g) for _ in range(2))
    big = 6e4 if dtype == "f16" else 1e30
    v[:, :, 1, :32] = big               # a column group that is constant and large, beside others of the usual size
    k[:, 100:, 0, 32:] = 0.25           # constant, within a group that varies before
    cache = kvc.KVCache(1, 2, d, [200], dtype, bits=4)
    cache.append(k.to(TDT[dtype]), v.to(TDT[dtype]), [200], np.zeros(200, np.uint8))
    q = torch.empty(1, 1, 2, d, dtype=TDT[dtype], device="cuda").normal_(generator=g)
    for scale in (0.1, -0.1, 0.0, 1e-30):
        got = cache.decode_attention_layers(q, scale)
        ref = reference(cache, 0, q, 200, range(200), scale, 0)
        for h in range(2):
            for a in range(0, d, 32):
                close4(got[:, 0, h, a:a + 32], ref[:, h, a:a + 32], f"scale {scale} head {h} columns {a}")
    close4(cache.decode_attention_layers(torch.zeros_like(q), 0.1)[:, 0], reference(cache, 0, q * 0, 200, range(200), 0.1, 0), "zero query")
    # logits of thousands: one row has all the weight (its neighbours in the order are far below it)
    z = torch.einsum("hd,hnd->hn", q[0, 0].double().cpu(), values(*stored(cache, 0, 200))[0])
    top = z.topk(2).values
    scale = 2000.0 / float((top[:, 0] - top[:, 1]).min())
    got = cache.decode_attention_layers(q, scale)[0, 0]
    rows = values(*stored(cache, 0, 200, "v"))[0]
    for h in range(2):
        close4(got[h], rows[h, int(z[h].argmax())], f"head {h}")


@pytest.mark.parametrize("d", [64, 80, 128])
def test_steps_back_to_back(d):
    """Steps whose calls follow each other at once give what they give one by one: append, decode, a drafted token taken back,
    another's decode, sequences replaced."""
    def run(wait):
        cache, g, _, _ = fill(3, 4, d, [200, 64, 333, 1], "f16", spare=200, rot=16, seed=4)
        outs = []
        for i in range(60):
            x, y = (torch.empty(3, 4, 4, d, dtype=torch.float16, device="cuda").normal_(generator=g) for _ in range(2))
            q = query(cache, g)
            calls = [lambda: cache.append(x, y, [1] * 4, np.zeros(4, np.uint8)), lambda: outs.append(cache.decode_attention_layers(q, 0.1)),
                     lambda: outs.append(cache.decode_attention_layers(q, 0.2))]
            if i % 3 == 0:
                back = cache.lengths()[0].copy()
                calls.append(lambda: cache.truncate(back))
                calls.append(lambda: outs.append(cache.decode_attention_layers(q, 0.1)))
            if i % 7 == 0:
                calls.append(lambda: cache.copy_from(cache, [3], [1]))
                calls.append(lambda: outs.append(cache.decode_attention_layers(q, 0.1)))
            for call in calls:
                call()
                if wait:
                    torch.cuda.synchronize()
        assert cache.device_status() == 0
        return outs

    for a, b in zip(run(False), run(True)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,sizes", [("f16", [1e4, 1e-3, 1.0, 30.0]), ("bf16", [1e20, 1e-20, 1.0, 1e-3])])
@pytest.mark.parametrize("d", [64, 80, 128])
def test_groups_of_different_sizes(d, dtype, sizes):
    """Each group of the output's columns to its own size, though the values' groups differ by many powers of two, and so in one
    part of a long sequence as in another."""
    n = 5003
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    k, v = (torch.empty(1, n, 2, d, device="cuda").normal_(generator=g) for _ in range(2))
    for i, a in enumerate(range(0, d, 32)):
        v[..., a:a + 32] *= sizes[i]
    cache = kvc.KVCache(1, 2, d, [n], dtype, bits=4)
    cache.append(k.to(TDT[dtype]), v.to(TDT[dtype]), [n], np.zeros(n, np.uint8))
    q = torch.empty(1, 1, 2, d, dtype=TDT[dtype], device="cuda").normal_(0, 2, generator=g)
    got = cache.decode_attention_layers(q, 0.125)
    ref = reference(cache, 0, q, n, range(n), 0.125, 0)
    for a in range(0, d, 32):
        close4(got[:, 0, :, a:a + 32], ref[:, :, a:a + 32], f"columns {a}")
