"""The decode over a cache of 4 bits on rows of the usual kind, near what its arithmetic leaves, and decodes of 16-bit caches after
copies to the bound of the other 16-bit decodes."""
import math

import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc
from _packed import CL, CR, fill
from _packed_usual import close_usual, expected
from _serving import attend, close, collected, make, query, rows_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rot", [0, 48])
def test_decode(d, dtype, rot):
    lens = [16, 65, 130, 511, 1000]
    cache, g, _, _ = fill(2, 8, d, lens, dtype, rot=rot, spare=1)
    q = query(cache, g, sd=1.0)
    scale = 1 / math.sqrt(d)
    got = cache.decode_attention_layers(q, scale)
    for s, n in enumerate(lens):
        close_usual(got[:, s], expected(cache, s, q, n, scale, pos=n - 1), f"{n} rows")


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (80, "bf16"), (96, "f16"), (128, "bf16")])
def test_decode_of_long_and_of_many_sequences(d, dtype):
    """What is left of the sums' halves falls with the root of the rows, and so the bound rises past a thousand."""
    scale = 1 / math.sqrt(d)
    cache, g, _, _ = fill(1, 4, d, [20011], dtype)
    q = query(cache, g, sd=1.0)
    got = cache.decode_attention_layers(q, scale)
    close_usual(got[:, 0], expected(cache, 0, q, 20011, scale), deviation=math.sqrt(20011 / 1000))
    lens = [200 + 37 * i for i in range(20)]
    cache, g, _, _ = fill(1, 32, d, lens, dtype)
    q = query(cache, g, sd=1.0)
    got = cache.decode_attention_layers(q, scale)
    for s in (0, 7, 19):
        close_usual(got[:, s], expected(cache, s, q, lens[s], scale), f"{lens[s]} rows")


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f16")])
def test_decode_with_hidden_rows(d, dtype):
    lens = [150, 300]
    kinds = [np.zeros(n, np.uint8) for n in lens]
    kinds[0][100] = CL
    kinds[1][70], kinds[1][140] = CL, CR
    cache, g, _, _ = fill(2, 8, d, lens, dtype, kinds=kinds)
    q = query(cache, g, sd=1.0)
    scale = 1 / math.sqrt(d)
    got = cache.decode_attention_layers(q, scale)
    for s, rows in enumerate(([i for i in range(150) if i != 100], [i for i in range(300) if not 70 <= i < 140])):
        close_usual(got[:, s], expected(cache, s, q, lens[s], scale, rows), f"sequence {s}")


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_decode_of_16_bits_after_copies_and_cuts(d, dtype):
    lens = [300, 0, 129, 0]
    cache, g = make(2, 3, d, lens, dtype, spare=400)
    cache.copy_from(cache, [1, 3], [0, 2])
    cache.truncate([-1, 257, -1, 70])
    now = [300, 257, 129, 70]
    q = query(cache, g)
    out = cache.decode_attention_layers(q, 0.1)
    for s, n in enumerate(now):
        k, v = rows_of(cache, s, n)
        assert torch.equal(k, rows_of(cache, s - s % 2, n)[0])
        for m in range(2):
            close(out[m, s], attend(q[m, s].double(), k[m], v[m], list(range(n)), 0.1)[0], f"sequence {s}")
