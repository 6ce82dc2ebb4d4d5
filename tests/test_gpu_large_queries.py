"""Rotated f16 queries near the type's largest value, whose turned columns lie above it: finite inputs have finite outputs
and weights.

A turned column past 65,504 goes into the products in steps of 16, off by 8 at most and by 4.6 in the mean square.  With C
such columns of a query, keys of deviation 1 and largest about 4.5, a logit in base e is off by 4.6 sqrt(C) SCALE =
7.0e-5 sqrt(C) in the mean square and by 8 sqrt(C) 4.5 SCALE at most (signs at random), a weight by as much of itself, and
a whole output or sum of weights by the mean square of its norm.  At most every third pair of columns is that large, and
one column of each: C <= d / 6 + 1 = 22 at 128 columns: 3.3e-4 of the norm, 2.6e-3 of a weight."""
import pytest
import torch

from _serving import collected  # noqa: F401
from _serving import attend, make, per_row, query, rotate, rows_of
from test_gpu_score_prompt import queries, reference
from test_gpu_shared_prefix import check, pair

pytestmark = pytest.mark.gpu

SCALE = 2.0 ** -16  # logits of a few units, as everywhere
NORM, WEIGHT = 3.3e-4, 2.6e-3


def off(got, ref):
    got, ref = got.double(), ref.double()
    assert torch.isfinite(got).all()
    return float((got - ref).norm() / ref.norm())


def large(q, rot):
    """Queries of deviation 2 / SCALE / sqrt(d), some columns and their partners at +-60,000."""
    d = q.shape[-1]
    q.mul_(2.0 ** 15 / d ** 0.5).clamp_(-60000, 60000)
    for i in range(0, rot // 2, 3):
        q[..., i], q[..., i + rot // 2] = 60000, (60000 if i % 2 else -60000)
    return q


@pytest.mark.parametrize("members", [4, 20, 40])
@pytest.mark.parametrize("d,rot", [(64, 64), (80, 32), (128, 128)])
def test_shared_decode(members, d, rot):
    parent, own = [0] * members, [2] * members
    prefix, cache, g = pair(1, 2, d, [300], parent, own, "f16", rot, seed=members)
    q = large(query(cache, g, sd=1.0), rot)
    out = cache.decode_attention_shared(q, SCALE)
    kp, vp = rows_of(prefix, 0, 300)
    for s in range(members):
        ko, vo = rows_of(cache, s, 2)
        k, v = torch.cat([kp[0], ko[0]], 1), torch.cat([vp[0], vo[0]], 1)
        ref, _ = attend(rotate(q[0, s], 301, rot), k, v, list(range(302)), SCALE)
        assert off(out[0, s], ref) <= NORM, s
    assert cache.device_status() == 0


@pytest.mark.parametrize("n_q", [12, 100, 300])
@pytest.mark.parametrize("d,rot", [(64, 64), (80, 32), (128, 128)])
def test_prompt_scores(n_q, d, rot):
    cache, g = make(1, 2, d, [300], "f16", rot, seed=n_q)
    q = large(queries(cache, [n_q], g, 1.0), rot)
    sc = cache.attach_scores()
    cache.score_prompt(0, q, [n_q], SCALE)
    ref = reference(cache, 0, 0, q, n_q, SCALE, cache.masked_reference_layout(0)["stored_pos"])
    got = per_row(cache, sc, 0, 300)[0]
    assert off(got, ref) <= NORM
    assert float(((got.double() - ref).abs() - WEIGHT * ref).max()) <= 1e-9
    assert cache.device_status() == 0


@pytest.mark.parametrize("d,rot", [(64, 32), (80, 16)])
def test_columns_that_are_not_turned_keep_their_smallest_values(d, rot):
    """Subnormal columns past the rotated ones."""
    parent, own = [0] * 4, [2] * 4
    prefix, cache, g = pair(1, 2, d, [300], parent, own, "f16", rot, seed=3)
    q = query(cache, g)
    q[..., rot:] = torch.randint(-15, 16, q[..., rot:].shape, generator=g, device="cuda").half() * 2.0 ** -24
    q[..., :rot] = 0
    out = cache.decode_attention_shared(q, 2.0 ** 18)
    check(prefix, cache, parent, own, q, 2.0 ** 18, out)
