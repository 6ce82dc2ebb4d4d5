"""The span book's side of an eviction, against a plain record of the rows (host only)."""
import numpy as np
import pytest

import paper_2310_08152_gb300 as kvc

N, CL, CR = kvc.NORMAL, kvc.CL, kvc.CR


@pytest.mark.parametrize("policy", [kvc.POLICY_PAPER, kvc.POLICY_KEEP_CL])
def test_random_histories(policy):
    rng = np.random.default_rng(11 + policy)
    for trial in range(60):
        book = kvc.Book(1, [100000], policy)
        rows, kinds, closed, cl_at = [], [], [], -1  # rows: history indices, -1 once unnamed
        for _ in range(40):
            act = rng.integers(0, 4)
            if act <= 1:
                new = []
                for _ in range(int(rng.integers(1, 12))):
                    k = N
                    if cl_at < 0 and rng.random() < 0.2:
                        k, cl_at = CL, len(kinds) + len(new)
                    elif cl_at >= 0 and rng.random() < 0.3:
                        closed.append((cl_at, len(kinds) + len(new)))
                        k, cl_at = CR, -1
                    new.append(k)
                book.append([len(new)], np.array(new, np.uint8))
                rows += range(len(kinds), len(kinds) + len(new))
                kinds += new
            elif act == 2 and closed:
                book.compress([0] * len(closed), *zip(*closed))
                for cl, cr in closed:
                    rows = [j for j in rows if not (cl + (policy != kvc.POLICY_PAPER) <= j < cr)]
                closed = []
            elif act == 3 and len(rows) > 3:
                keep = int(rng.integers(1, len(rows)))
                recent = int(rng.integers(1, keep + 1))
                first = next((j for j in rows[len(rows) - recent:] if j >= 0), len(kinds))
                spans = [c for c, _ in closed] + ([cl_at] if cl_at >= 0 else [])
                if any(c < first for c in spans):
                    with pytest.raises(kvc.KvcError) as e:
                        book.evict(keep, recent)
                    assert e.value.status == 5
                else:
                    book.evict(keep, recent)
                    rows = [-1] * (keep - recent) + rows[len(rows) - recent:]
            lay = book.layout(0)
            assert lay["stored_orig"].tolist() == rows
            assert lay["kinds"].tolist() == kinds
            assert book.lengths()[0][0] == len(rows)
            named = [j for j in rows if j >= 0]
            assert [p for p, j in zip(lay["stored_pos"], rows) if j >= 0] == lay["pos"][named].tolist()
            assert np.all(lay["stored_pos"][:len(rows) - len(named)] == -1)
            if kinds:
                vis = lay["visible"]
                first = named[0] if named else len(kinds)
                if kinds[-1] != CR:  # the query of a <CR> sees its interior even after that is freed
                    assert not vis[:first].any()
                # the decode attends to the unnamed rows and the visible named ones
                if kinds[-1] == CL:
                    assert book.lengths()[1][0] == 1
                elif not closed and kinds[-1] != CR:
                    assert book.lengths()[1][0] == len(rows) - len(named) + int(vis[named].sum())


def test_refusals():
    book = kvc.Book(2, [100, 100])
    book.append([50, 20], np.zeros(70, np.uint8))
    for keep, recent in (([10, 10], [11, 1]), ([10, 10], [1, 0]), ([0, 5], [1, 1])):
        with pytest.raises(kvc.KvcError) as e:
            book.evict(keep, recent)
        assert e.value.status == 1
    assert book.lengths()[0].tolist() == [50, 20]
    book.evict([30, -1], [4, 0])
    assert book.lengths()[0].tolist() == [30, 20]
    book.evict(25, 4)
    assert book.lengths()[0].tolist() == [25, 20]
    with pytest.raises(ValueError):
        book.evict([1, 2, 3], 1)
    local = kvc.Book(1, [100], kvc.POLICY_LOCAL, local_ratio=0.5)
    local.append([10], np.zeros(10, np.uint8))
    with pytest.raises(kvc.KvcError) as e:
        local.evict(5, 1)
    assert e.value.status == 2


def test_prefill_bounds_after_an_eviction():
    book = kvc.Book(1, [1000])
    book.append([100], np.zeros(100, np.uint8))
    book.evict(40, 10)
    kinds = np.array([N, CL, N, N, CR, N], np.uint8)
    book.append([6], kinds)
    meta = book.prefill_keys(0, 16)
    assert meta.size == 46
    hid = meta >> 1
    assert (hid[:41] == 0x3FFFFFFF).all() and hid[41] == 41 and (hid[42:44] == 44).all() and (hid[44:] == 0x3FFFFFFF).all()
    with pytest.raises(kvc.KvcError) as e:
        book.prefill_keys(0, 17)
    assert e.value.status == 5
