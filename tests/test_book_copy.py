"""The span book's side of copies and cuts, against books that never had the tokens, and refusals (host only)."""
import numpy as np
import pytest

import paper_2310_08152_gb300 as kvc

N, CL, CR = kvc.NORMAL, kvc.CL, kvc.CR


def same(a, s, b, t):
    x, y = a.layout(s), b.layout(t)
    for key in x:
        assert x[key].tolist() == y[key].tolist(), key
    assert a.pending_spans(s) == b.pending_spans(t)
    (la, aa), (lb, ab) = a.lengths(), b.lengths()
    assert (la[s], aa[s]) == (lb[t], ab[t])
    # the next tokens' positions, and that the spans are as open in both
    for k in ([N, N], [CL, N], [CR, N]):
        res = []
        for book, at in ((a, s), (b, t)):
            n_new = np.zeros(book.b, np.int32)
            n_new[at] = 2
            try:
                res.append(book.next_positions(n_new, np.array(k, np.uint8)).tolist())
            except kvc.KvcError as e:
                res.append(e.status)
        assert res[0] == res[1], k


def history(rng, n):
    kinds, cl, spans = [], -1, []
    for j in range(n):
        k = N
        if cl < 0 and rng.random() < 0.15:
            k, cl = CL, j
        elif cl >= 0 and rng.random() < 0.25:
            k = CR
            spans.append((cl, j))
            cl = -1
        kinds.append(k)
    return kinds, spans


@pytest.mark.parametrize("policy", [kvc.POLICY_PAPER, kvc.POLICY_KEEP_CL])
def test_cut_equals_never_appended(policy):
    rng = np.random.default_rng(5 + policy)
    for trial in range(80):
        n = int(rng.integers(2, 60))
        kinds, spans = history(rng, n)
        freed = [sp for sp in spans if rng.random() < 0.6]
        book = kvc.Book(2, [1000, 1000], policy)
        book.append([n, 3], np.array(kinds + [N] * 3, np.uint8))
        if freed:
            book.compress([0] * len(freed), *zip(*freed))
        cut = int(rng.integers(1, n + 1))
        before = book.layout(0)
        if any(a < cut <= z for a, z in freed):
            with pytest.raises(kvc.KvcError) as e:
                book.truncate([cut, -1])
            assert e.value.status == 5
            after = book.layout(0)
            assert all(before[k].tolist() == after[k].tolist() for k in before)
            continue
        book.truncate([cut, -1])
        plain = kvc.Book(2, [1000, 1000], policy)
        plain.append([cut, 3], np.array(kinds[:cut] + [N] * 3, np.uint8))
        kept = [sp for sp in freed if sp[1] < cut]
        if kept:
            plain.compress([0] * len(kept), *zip(*kept))
        same(book, 0, plain, 0)
        same(book, 1, plain, 1)
        # and they go on alike
        more = [N, N, N]
        for b in (book, plain):
            b.append([3, 0], np.array(more, np.uint8))
        same(book, 0, plain, 0)


def test_free_and_cut_of_an_evicted_sequence():
    book = kvc.Book(1, [100], kvc.POLICY_PAPER)
    book.append([40], np.zeros(40, np.uint8))
    book.evict(20, 5)  # rows of tokens 35 .. 39 have names, 15 rows have none
    with pytest.raises(kvc.KvcError) as e:
        book.truncate(34)
    assert e.value.status == 5
    book.truncate(37)
    assert book.lengths()[0].tolist() == [17]
    assert book.layout(0)["stored_orig"].tolist() == [-1] * 15 + [35, 36]
    book.append([2], np.zeros(2, np.uint8))
    assert book.layout(0)["stored_orig"].tolist() == [-1] * 15 + [35, 36, 37, 38]
    book.truncate(0)
    assert book.lengths()[0].tolist() == [0]
    fresh = kvc.Book(1, [100], kvc.POLICY_PAPER)
    for b in (book, fresh):
        b.append([4], np.array([CL, N, CR, N], np.uint8))
    same(book, 0, fresh, 0)


def test_cut_refusals():
    book = kvc.Book(2, [10, 10], kvc.POLICY_PAPER)
    book.append([4, 2], np.zeros(6, np.uint8))
    for bad, status in (([5, -1], 1), ([2, 3], 1)):
        with pytest.raises(kvc.KvcError) as e:
            book.truncate(bad)
        assert e.value.status == status
        assert book.lengths()[0].tolist() == [4, 2]
    book.truncate([4, -7])  # nothing to drop
    assert book.lengths()[0].tolist() == [4, 2]
    ring = kvc.Book(1, [4], kvc.POLICY_LOCAL, local_ratio=0.5)
    ring.append([6], np.zeros(6, np.uint8))
    with pytest.raises(kvc.KvcError) as e:
        ring.truncate(5)
    assert e.value.status == 2
    ring.truncate(0)
    assert ring.lengths()[0].tolist() == [0]


@pytest.mark.parametrize("policy", [kvc.POLICY_PAPER, kvc.POLICY_KEEP_CL])
def test_copies(policy):
    rng = np.random.default_rng(9)
    kinds, spans = history(rng, 50)
    a = kvc.Book(4, [60] * 4, policy)
    a.append([50, 7, 0, 0], np.array(kinds + [N] * 7, np.uint8))
    a.compress([0], [spans[0][0]], [spans[0][1]])
    b = kvc.Book(3, [55, 80, 60], policy)
    b.append([0, 9, 2], np.zeros(11, np.uint8))
    b.copy_from(a, [2, 0], [0, 0])
    same(b, 2, a, 0)
    same(b, 0, a, 0)
    a.copy_from(a, [3, 2], [1, 0])
    same(a, 3, a, 1)
    same(a, 2, a, 0)
    a.copy_from(b, [0], [1])  # over a longer one
    same(a, 0, b, 1)
    # copies go their own ways
    b.append([1, 0, 0], np.zeros(1, np.uint8))
    assert b.lengths()[0][0] == b.lengths()[0][2] + 1
    empty = kvc.Book(1, [5], policy)
    a.copy_from(empty, [3], [0])
    assert a.lengths()[0][3] == 0


def test_copy_refusals():
    a = kvc.Book(3, [20, 20, 4], kvc.POLICY_PAPER)
    a.append([5, 2, 0], np.zeros(7, np.uint8))
    other = kvc.Book(1, [20], kvc.POLICY_KEEP_CL)
    ring = kvc.Book(1, [20], kvc.POLICY_LOCAL, local_ratio=0.5)
    for book, dst, src, status in ((a, [2], [0], 3),        # capacity
                                   (a, [1, 1], [0, 0], 1),  # a target twice
                                   (a, [1, 0], [0, 2], 1),  # a target and a source
                                   (a, [0], [0], 1),
                                   (a, [3], [0], 1), (a, [-1], [0], 1), (a, [1], [3], 1), (a, [1], [-1], 1),
                                   (other, [1], [0], 1), (ring, [1], [0], 2)):
        with pytest.raises(kvc.KvcError) as e:
            a.copy_from(book, dst, src)
        assert e.value.status == status, (dst, src)
        assert a.lengths()[0].tolist() == [5, 2, 0]
    with pytest.raises(ValueError):
        a.copy_from(a, [1, 2], [0])
    a.copy_from(a, [], [])


def handle(bits=4, d=64, policy=kvc.POLICY_PAPER, M=2, H=8, rot=0, dtype="f16"):
    """A cache's handle with buffers that nothing touches."""
    cfg, _ = kvc.make_config(M, H, d, [16, 7], dtype, rot, 10000.0, policy, 0.5, bits)
    cfg.k_base = cfg.v_base = cfg.pos_base = cfg.orig_base = cfg.workspace = 1 << 40
    cfg.workspace_bytes = 1 << 40
    return kvc.kvc_create(cfg)


class Buffer:
    def data_ptr(self):
        return 1 << 41


def test_calls_that_need_16_bits():
    c, wide = handle(), handle(16)
    n = np.zeros(2, np.int32)
    calls = [lambda: kvc.kvc_set_scores(c, Buffer()), lambda: kvc.kvc_score_scratch_bytes(c, n), lambda: kvc.kvc_evict(c, [1, 1], [1, 1], stream=0),
             lambda: kvc.kvc_prefill_attention(c, 0, Buffer(), n, 1.0, Buffer(), stream=0)]
    calls += [lambda x=x, y=y: kvc.lib().kvc_set_prefix(x, y, np.zeros(2, np.int32).ctypes.data, 1 << 41, 1 << 40)
              for x, y in ((c, wide), (wide, c))]
    for i, call in enumerate(calls):
        try:
            rc = call()
        except kvc.KvcError as e:
            rc = e.status
        assert rc == 2, i
    kvc.kvc_set_scores(c, None)
    for h in (c, wide):
        kvc.kvc_destroy(h)


def test_config_and_sizes_of_4_bits():
    for bad in (8, 3, -4):
        with pytest.raises(kvc.KvcError) as e:
            handle(bad)
        assert e.value.status == 2
    with pytest.raises(kvc.KvcError) as e:
        handle(4, policy=kvc.POLICY_LOCAL)
    assert e.value.status == 2
    for d, groups in ((64, 2), (80, 3), (96, 3), (128, 4)):
        cfg, _ = kvc.make_config(2, 3, d, [16, 7, 1], bits=4)
        sizes = kvc.kvc_required_bytes(cfg)
        rows = 2 * 3 * (16 + 8 + 4)  # capacities rounded up to multiples of 4
        codes = (rows * d // 2 + 255) // 256 * 256
        assert sizes["k"] == sizes["v"] == codes + rows * groups * 4
        assert sizes["meta"] == 4 * 28
        wide, _ = kvc.make_config(2, 3, d, [16, 7, 1], bits=0)
        assert kvc.kvc_required_bytes(wide)["k"] == 2 * 3 * 24 * d * 2


def test_copy_and_cut_of_caches_without_rows():
    """What is refused before any device work."""
    a, b = handle(), handle(16)
    for other, status in ((handle(16, d=80), 1), (handle(4, M=1), 1), (handle(4, H=4), 1), (handle(4, rot=16), 1),
                          (handle(4, dtype="bf16"), 1), (handle(16, policy=kvc.POLICY_KEEP_CL), 1)):
        with pytest.raises(kvc.KvcError) as e:
            kvc.kvc_copy(a, other, [0], [0], stream=0)
        assert e.value.status == status
        kvc.kvc_destroy(other)
    for dst, src in (([0, 0], [0, 1]), ([2], [0]), ([0], [2])):
        with pytest.raises(kvc.KvcError) as e:
            kvc.kvc_copy(a, b, dst, src, stream=0)
        assert e.value.status == 1
    with pytest.raises(kvc.KvcError) as e:
        kvc.kvc_copy(a, a, [0], [0], stream=0)
    assert e.value.status == 1
    kvc.kvc_copy(a, b, [], [], stream=0)
    with pytest.raises(kvc.KvcError) as e:
        kvc.kvc_truncate(a, [1, 0], stream=0)
    assert e.value.status == 1
    kvc.kvc_truncate(a, [0, -1], stream=0)
    L = kvc.lib()
    assert L.kvc_copy(None, a, 0, None, None, None) == 1 and L.kvc_copy(a, None, 0, None, None, None) == 1
    assert L.kvc_copy(a, b, 1, None, None, None) == 1 and L.kvc_copy(a, b, -1, None, None, None) == 1
    assert L.kvc_truncate(None, None, None) == 1 and L.kvc_truncate(a, None, None) == 1
    assert L.kvc_book_truncate(None, None) == 1 and L.kvc_book_copy(None, None, 0, None, None) == 1
    for h in (a, b):
        kvc.kvc_destroy(h)
