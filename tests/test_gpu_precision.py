"""How near 64 bits the shared decode and the prompt scores come: nearer than 16-bit parts that are too few, sums that the
tensor cores cut too often, or approximate angles would leave them.

With q of deviation 2 and K of 1 a logit in the base-2 exponent has deviation 2.9, and the rows that count lie below 16,
where a sum's last bit is 2^-20.  The tensor cores cut there in each of the d / 16 steps of the largest part, which leaves
2^-20 / sqrt(12) sqrt(d / 16) ln 2 = 5.4e-7 of a weight at 128 columns (what is common to all rows cancels).  Besides: the
exponential, to 2^-22, 1.4e-7; a rotated f16 query of 22 bits, 2.4e-7; P of 22 bits or more, 0.7e-7; products with V cut in
sums of up to 128 rows, 2e-7, and those sums added in 32 bits, 5,000 rows 16 at a time, 3.2e-7.  Together 7.3e-7 of an
output's norm (independent errors); NORM is twice that.  Weights summed over queries have less."""
import pytest
import torch

from _serving import collected  # noqa: F401
from _serving import attend, make, per_row, query, rotate, rows_of
from test_gpu_score_prompt import queries, reference
from test_gpu_shared_prefix import pair

pytestmark = pytest.mark.gpu

NORM = 1.45e-6
TYPES = [(64, "f16", 0), (64, "f16", 64), (64, "bf16", 64), (80, "bf16", 80), (96, "f16", 96), (96, "bf16", 0), (128, "f16", 128),
         (128, "bf16", 0), (128, "bf16", 128)]


def shared_error(d, dtype, rot, n, members, M=1, H=2, own=2):
    """The shared decode's error over two heads of the first and the last layer and eight members."""
    prefix, cache, g = pair(M, H, d, [n], [0] * members, [own] * members, dtype, rot, seed=d + members)
    q = query(cache, g)
    out = cache.decode_attention_shared(q, d ** -0.5)
    kp, vp = rows_of(prefix, 0, n)
    num = den = 0.0
    for m in {0, M - 1}:
        for s in range(0, members, (members + 7) // 8):
            ko, vo = rows_of(cache, s, own)
            k, v = torch.cat([kp[m], ko[m]], 1)[:2], torch.cat([vp[m], vo[m]], 1)[:2]
            ref, _ = attend(rotate(q[m, s, :2], n + own - 1, rot), k, v, list(range(n + own)), d ** -0.5)
            num += float((out[m, s, :2].double() - ref).norm() ** 2)
            den += float(ref.norm() ** 2)
    return (num / den) ** 0.5


@pytest.mark.parametrize("d,dtype,rot", TYPES)
@pytest.mark.parametrize("members", [8, 24, 40, 130])
def test_shared_decode(members, d, dtype, rot):
    assert shared_error(d, dtype, rot, 5000, members) <= NORM


@pytest.mark.parametrize("d,dtype,rot", [(64, "f16", 64), (80, "bf16", 0), (128, "bf16", 128)])
@pytest.mark.parametrize("members", [24, 40])
def test_shared_decode_of_whole_prefixes(members, d, dtype, rot):
    """Heads and layers enough that a prefix is one run."""
    assert shared_error(d, dtype, rot, 5000, members, 10, 32) <= NORM


@pytest.mark.parametrize("d,dtype,rot", TYPES)
@pytest.mark.parametrize("n,n_q", [(3000, 12), (3000, 64), (3000, 100), (1500, 1500)])
def test_prompt_scores(n, n_q, d, dtype, rot):
    cache, g = make(1, 2, d, [n], dtype, rot, seed=d)
    q = queries(cache, [n_q], g)
    sc = cache.attach_scores()
    cache.score_prompt(0, q, [n_q], d ** -0.5)
    ref = reference(cache, 0, 0, q, n_q, d ** -0.5, cache.masked_reference_layout(0)["stored_pos"])
    got = per_row(cache, sc, 0, n)[0].double()
    assert float((got - ref).norm() / ref.norm()) <= NORM
