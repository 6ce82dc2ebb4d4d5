"""Eviction by accumulated attention weight: rows, scores, metadata and what works after it."""
import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc

from _serving import collected  # noqa: F401
from _serving import attend, close, evict_reference, make, per_row, query, rows_of

pytestmark = pytest.mark.gpu


def fill(cache, lens, make_scores):
    for s, n in enumerate(lens):
        if n:
            per_row(cache, cache.scores, s, n).copy_(make_scores(s, n))


def evict_and_check(cache, lens, keep, recent):
    """Evicts and compares every stream with the reference; the lengths after it."""
    keep, recent = np.broadcast_to(keep, (cache.b,)), np.broadcast_to(recent, (cache.b,))
    old = [(rows_of(cache, s, n)[0].clone(), rows_of(cache, s, n)[1].clone(), per_row(cache, cache.scores, s, n).clone(),
            cache.masked_reference_layout(s)) for s, n in enumerate(lens)]
    kept = torch.full((cache.M, cache.H * cache.C), -7, dtype=torch.int32, device="cuda")
    cache.evict(keep, recent, kept=kept)
    after = []
    for s, n in enumerate(lens):
        k0, v0, s0, lay0 = old[s]
        untouched = keep[s] < 0 or n <= keep[s]
        n1 = n if untouched else int(keep[s])
        after.append(n1)
        k1, v1 = rows_of(cache, s, n1)
        s1, kp = per_row(cache, cache.scores, s, int(cache.capacity[s])), per_row(cache, kept, s, n1)
        lay = cache.masked_reference_layout(s)
        assert lay["stored_orig"].size == n1
        if untouched:
            assert torch.equal(k1, k0) and torch.equal(v1, v0) and torch.equal(s1[:, :, :n], s0) and torch.all(kp == -7)
            assert np.array_equal(lay["stored_orig"], lay0["stored_orig"])
            continue
        sc = s0.cpu().numpy()
        for m in range(cache.M):
            for h in range(cache.H):
                ref = torch.tensor(evict_reference(sc[m, h].tolist(), n1, int(recent[s])), device="cuda")
                what = f"sequence {s}, layer {m}, head {h}"
                assert torch.equal(kp[m, h].long(), ref), what
                assert torch.equal(k1[m, h].view(torch.int16), k0[m, h][ref].view(torch.int16)), what
                assert torch.equal(v1[m, h].view(torch.int16), v0[m, h][ref].view(torch.int16)), what
                assert torch.equal(s1[m, h, :n1].view(torch.int32), s0[m, h][ref].view(torch.int32)), what
        assert torch.all(s1[:, :, n1:] == 0)
        r = int(recent[s])
        assert np.all(lay["stored_orig"][:n1 - r] == -1) and np.all(lay["stored_pos"][:n1 - r] == -1)
        assert np.array_equal(lay["stored_orig"][n1 - r:], lay0["stored_orig"][n - r:])
        assert np.array_equal(lay["stored_pos"][n1 - r:], lay0["stored_pos"][n - r:])
        book = cache.book.layout(s)
        assert np.array_equal(book["stored_orig"], lay["stored_orig"]) and np.array_equal(book["stored_pos"], lay["stored_pos"])
    assert list(cache.lengths()[0]) == after
    assert cache.device_status() == 0
    return after


def spread(s, n, M=2, H=3):
    return torch.randn(M, H, n, device="cuda").mul_(2).exp_()


CASES = [(2, 1, 1), (3, 2, 1), (10, 4, 2), (100, 99, 7), (100, 64, 64), (1000, 400, 30), (1025, 1024, 1), (2000, 1, 1),
         (2000, 1999, 1999), (3000, 1500, 1400), (5000, 1237, 100), (9000, 8000, 64)]


@pytest.mark.parametrize("n,keep,recent", CASES)
@pytest.mark.parametrize("d,dtype", [(64, "f16"), (80, "bf16"), (96, "f16"), (128, "bf16")])
def test_sizes(n, keep, recent, d, dtype):
    cache, _ = make(2, 3, d, [n], dtype, seed=n + d)
    cache.attach_scores()
    torch.manual_seed(n)
    fill(cache, [n], spread)
    evict_and_check(cache, [n], keep, recent)


@pytest.mark.parametrize("n", [500, 3333])
@pytest.mark.parametrize("kind", ["equal", "few values", "zeros and ones", "nan and inf", "negative", "tiny", "rising", "falling"])
def test_ties_and_odd_scores(kind, n):
    def scores(s, n):
        x = torch.rand(2, 3, n, device="cuda")
        if kind == "equal":
            return torch.full_like(x, 0.25)
        if kind == "few values":
            return (x * 5).floor()
        if kind == "zeros and ones":
            return torch.where(x < 0.5, torch.where(x < 0.25, 0.0, -0.0), 1.0)
        if kind == "nan and inf":
            x[:, :, ::7] = float("nan")
            x[:, :, 3::11] = float("inf")
            x[:, :, 5::13] = float("-inf")
            return x
        if kind == "negative":
            return x - 0.5
        if kind == "tiny":
            return x * 1e-42
        return torch.arange(n, device="cuda").float().mul(1 if kind == "rising" else -1).expand(2, 3, n)

    torch.manual_seed(1)
    for keep, recent in ((n // 2, 17), (n - 1, 1), (n // 5, n // 10)):
        cache, _ = make(2, 3, 64, [n])
        cache.attach_scores()
        fill(cache, [n], scores)
        evict_and_check(cache, [n], keep, recent)


def test_ragged_budgets_and_sequences_left_alone():
    lens = [700, 0, 64, 1, 1500, 300]
    cache, _ = make(2, 3, 80, lens)
    cache.attach_scores()
    fill(cache, lens, spread)
    evict_and_check(cache, lens, [100, 5, 64, 1, 600, -1], [10, 1, 3, 1, 600, -5])


def test_many_streams():
    cache, _ = make(8, 32, 64, [300, 520, 90])
    cache.attach_scores()
    fill(cache, [300, 520, 90], lambda s, n: spread(s, n, 8, 32))
    evict_and_check(cache, [300, 520, 90], 80, 16)


@pytest.mark.parametrize("drop", [1, 40])
def test_large_batch(drop):
    """A plan too large for a kernel parameter."""
    lens = [60 + s % 7 + drop for s in range(130)]
    cache, _ = make(1, 2, 64, lens)
    cache.attach_scores()
    fill(cache, lens, lambda s, n: spread(s, n, 1, 2))
    evict_and_check(cache, lens, 60, 11)
    q = query(cache, torch.Generator(device="cuda"))
    out = cache.decode_attention_layers(q, 0.125)  # the state that later calls read went up with the plan
    for s in (0, 77, 129):
        k, v = rows_of(cache, s, 60)
        close(out[0, s], attend(q[0, s].double(), k[0], v[0], list(range(60)), 0.125)[0])


def test_candidates_that_do_not_fit_shared_memory():
    n = 50001
    cache, _ = make(1, 2, 64, [n])
    cache.attach_scores()
    fill(cache, [n], lambda s, n: torch.rand(1, 2, n, device="cuda").mul(3000).floor())
    evict_and_check(cache, [n], 20000, 333)


def test_generation_goes_on_after_evictions():
    """Appends, scored decodes, spans and evictions in turn, against a plain record of every stream's rows."""
    M, H, d, b = 2, 3, 64, 2
    N, CL, CR = kvc.NORMAL, kvc.CL, kvc.CR
    rng = np.random.default_rng(0)
    lens = [90, 61]
    cache, g = make(M, H, d, lens, spare=80)
    cache.attach_scores()
    K = [rows_of(cache, s, n)[0].clone() for s, n in enumerate(lens)]
    V = [rows_of(cache, s, n)[1].clone() for s, n in enumerate(lens)]
    S = [torch.zeros(M, H, n, dtype=torch.float64, device="cuda") for n in lens]
    open_at = [-1, -1]  # stored row of the open <CL>
    for step in range(60):
        kinds = []
        for s in range(b):
            k = N
            if open_at[s] < 0 and rng.random() < 0.15:
                k = CL
            elif open_at[s] >= 0 and rng.random() < 0.3:
                k = CR
            kinds.append(k)
        new = torch.empty(2, M, b, H, d, dtype=torch.float16, device="cuda").normal_(generator=g)
        cache.append(new[0], new[1], [1] * b, kinds)
        q = query(cache, g)
        out = cache.decode_attention_scored(q, 0.125)
        for s in range(b):
            K[s], V[s] = (torch.cat([x, y[:, s][:, :, None]], 2) for x, y in ((K[s], new[0]), (V[s], new[1])))
            n = K[s].shape[2]
            if kinds[s] == CL:
                seen, open_at[s] = [n - 1], n - 1
            else:
                seen = [i for i in range(n) if i != open_at[s]]
            S[s] = torch.cat([S[s], torch.zeros(M, H, 1, dtype=torch.float64, device="cuda")], 2)
            for m in range(M):
                ref, w = attend(q[m, s].double(), K[s][m], V[s][m], seen, 0.125)
                close(out[m, s], ref, f"step {step} sequence {s} layer {m}")
                S[s][m][:, seen] += w
            got = per_row(cache, cache.scores, s, n)
            assert (got.double() - S[s]).abs().max() <= 1e-5 * (1 + S[s].max())
            S[s] = got.double().clone()  # further steps start from the cache's own scores
        for s in range(b):
            if kinds[s] == CR:
                cl, cr = cache.pending_spans(s)[-1]
                cache.compress_spans([s], [cl], [cr])
                rows = [i for i in range(K[s].shape[2]) if i < open_at[s] or i == K[s].shape[2] - 1]
                K[s], V[s], S[s] = K[s][:, :, rows], V[s][:, :, rows], S[s][:, :, rows]
                open_at[s] = -1
        if step % 7 == 6:
            keep = [min(60, K[s].shape[2]) if open_at[s] < 0 else -1 for s in range(b)]
            n0 = [K[s].shape[2] for s in range(b)]
            cache.evict(keep, [20] * b)
            for s in range(b):
                if keep[s] < 0 or n0[s] <= keep[s]:
                    continue
                sc = S[s].float().cpu().numpy()
                at = torch.tensor([[evict_reference(sc[m, h].tolist(), keep[s], 20) for h in range(H)] for m in range(M)],
                                  device="cuda")
                S[s] = S[s].gather(2, at)
                i = at[..., None].expand(M, H, keep[s], d)
                K[s], V[s] = K[s].gather(2, i), V[s].gather(2, i)
        for s in range(b):
            k, v = rows_of(cache, s, K[s].shape[2])
            assert torch.equal(k, K[s]) and torch.equal(v, V[s]), (step, s)
    assert cache.device_status() == 0


def test_prefill_of_later_tokens():
    cache, g = make(1, 2, 64, [300], spare=100)
    cache.attach_scores()
    fill(cache, [300], lambda s, n: torch.rand(1, 2, n, device="cuda"))
    evict_and_check(cache, [300], 120, 30)
    new = torch.empty(2, 1, 50, 2, 64, dtype=torch.float16, device="cuda").normal_(generator=g)
    cache.append(new[0], new[1], [50], np.zeros(50, np.uint8))
    q = torch.empty(50, 2, 64, dtype=torch.float16, device="cuda").normal_(generator=g)
    out = cache.prefill_attention(0, q, [50], 0.125)
    k, v = rows_of(cache, 0, 170)
    for t in range(50):
        ref, _ = attend(q[t].double(), k[0], v[0], list(range(121 + t)), 0.125)
        assert (out[t].double() - ref).abs().max() <= 2e-3
    with pytest.raises(kvc.KvcError) as e:  # the 81st token from the end is one of the unnamed rows
        cache.prefill_attention(0, torch.zeros(81, 2, 64, dtype=torch.float16, device="cuda"), [81], 0.125)
    assert e.value.status == 5


def test_refusals():
    N, CL, CR = kvc.NORMAL, kvc.CL, kvc.CR
    kinds = [np.array([N] * 30 + [CL] + [N] * 10, np.uint8)]
    cache, _ = make(1, 2, 64, [41], kinds=kinds, spare=3)
    with pytest.raises(kvc.KvcError) as e:
        cache.evict(20, 5)
    assert e.value.status == 5  # no scores
    cache.attach_scores()
    for keep, recent in ((20, 0), (20, 21), (0, 0)):
        with pytest.raises(kvc.KvcError) as e:
            cache.evict(keep, recent)
        assert e.value.status == 1, (keep, recent)
    with pytest.raises(kvc.KvcError) as e:  # the open span is older than the recent rows
        cache.evict(20, 10)
    assert e.value.status == 5 and cache.lengths()[0][0] == 41
    with pytest.raises(ValueError):
        cache.evict([20, 20], 5)
    with pytest.raises(ValueError):
        cache.evict(20, 11, kept=torch.zeros(3, dtype=torch.int32, device="cuda"))
    cache.evict(20, 11)
    assert cache.lengths()[0][0] == 20
    new = torch.zeros(1, 2, 64, dtype=torch.float16, device="cuda")
    cache.append(new, new, [1], [CR])
    with pytest.raises(kvc.KvcError) as e:  # closed, and not freed
        cache.evict(15, 3)
    assert e.value.status == 5
    cache.compress_spans([0], [30], [41])
    assert cache.lengths()[0][0] == 10
    cache.evict(5, 1)
    assert cache.device_status() == 0
