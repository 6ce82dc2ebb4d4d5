"""The decode over a cache of 4 bits where the size of a group of columns of the values changes along a sequence: each group's
outputs are held to their own size, and to what rows of the usual kind allow."""
import math

import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc
from _packed_usual import close_groups, expected
from _serving import TDT, collected  # noqa: F401

pytestmark = pytest.mark.gpu

LOWEST = {"f16": 1e-6, "bf16": 1e-30}  # sizes whose steps the type holds


ONE, MANY = 1, 640  # segments: pieces of a tile each (their tiles are fewer than the GPU's workers), or of several tiles


def decode(size, d, dtype, segments=MANY, key_size=None, seed=1, deviation=1.0, what=""):
    """Values of deviation size [n, groups], keys of deviation key_size [n] (1), the same for every head and sequence."""
    n = size.shape[0]
    H = 1 if segments == 1 else 40
    b = max(1, segments * 1024 // n // H)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    k, v = (torch.empty(1, b, n, H, d, device="cuda").normal_(generator=g) for _ in range(2))
    if key_size is not None:
        k *= key_size.float().cuda()[None, None, :, None, None]
    v *= size.float().cuda().repeat_interleave(32, -1)[:, :d][None, None, :, None]
    cache = kvc.KVCache(1, H, d, [n] * b, dtype, bits=4)
    cache.append(*(x.to(TDT[dtype]).flatten(1, 2) for x in (k, v)), [n] * b, np.zeros(b * n, np.uint8))
    q = torch.empty(1, b, H, d, device="cuda").normal_(generator=g).to(TDT[dtype])
    scale = 1 / math.sqrt(d)
    got = cache.decode_attention_layers(q, scale)
    assert cache.device_status() == 0
    for s in sorted({0, b - 1}):
        close_groups(got[:, s], expected(cache, s, q, n, scale), what, deviation)


def groups(d):
    return (d + 31) // 32


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype,first", [("f16", 1e-5), ("f16", 1e-6), ("f16", 0.0), ("bf16", 1e-6), ("bf16", 1e-8), ("bf16", 1e-12),
                                         ("bf16", 1e-30), ("bf16", 0.0)])
@pytest.mark.parametrize("segments", [ONE, MANY])
def test_a_group_that_grows_after_the_first_rows(d, dtype, first, segments):
    size = torch.ones(1024, groups(d))
    for a in range(0, 1024, 320):  # wherever a worker's piece begins
        size[a:a + 64, 0] = first
    decode(size, d, dtype, segments)
    size[64:, 0] = 1.0
    decode(size, d, dtype, segments)


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_group_that_is_zero_and_then_tiny(d, dtype):
    size = torch.ones(1000, groups(d))
    size[:64, -1] = 0.0
    size[64:, -1] = LOWEST[dtype]
    decode(size, d, dtype)
    size[:, -1] = LOWEST[dtype]
    size[64:640, -1] = 0.0
    decode(size, d, dtype)


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("up", [True, False])
def test_sizes_that_change_row_by_row(d, dtype, up):
    """One group grows or shrinks steadily while the next does the opposite, over all that the type holds."""
    n, top = 3000, 1e3 if dtype == "f16" else 1e30
    run = torch.logspace(math.log10(LOWEST[dtype]), math.log10(top), n, dtype=torch.float64)
    size = torch.ones(n, groups(d), dtype=torch.float64)
    size[:, 0], size[:, 1] = (run, run.flip(0)) if up else (run.flip(0), run)
    decode(size, d, dtype)


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("seed", [3, 4])
def test_sizes_and_weights_that_wander(d, dtype, seed):
    """Groups' sizes by tile, and logits of a deviation that differs by row: the greatest products come from any of the rows."""
    n = 2500
    g = torch.Generator().manual_seed(seed)
    low, top = math.log10(LOWEST[dtype]), 3.0 if dtype == "f16" else 25.0
    size = 10.0 ** (low + (top - low) * torch.rand((n + 63) // 64, groups(d), generator=g, dtype=torch.float64))
    key = 8.0 * torch.rand(n, generator=g) ** 2
    decode(size.repeat_interleave(64, 0)[:n], d, dtype, key_size=key, seed=seed, deviation=8.0)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("at", [0, 500, 999])
@pytest.mark.parametrize("H", [1, 640])
def test_a_row_with_nearly_all_the_weight_has_none_of_a_group(d, dtype, at, H):
    """The group's columns are the other rows', whose weights are some 2^-40 together."""
    n = 1000
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    k, v = (torch.empty(1, n, H, d, device="cuda").normal_(generator=g) for _ in range(2))
    q = torch.empty(1, 1, H, d, device="cuda").normal_(generator=g).to(TDT[dtype])
    k[0, at] = 40 * q[0, 0].float() / q[0, 0].float().norm(dim=-1, keepdim=True) * math.sqrt(d) / q[0, 0].float().norm(dim=-1, keepdim=True)
    v[0, at, :, :32] = 0.0
    cache = kvc.KVCache(1, H, d, [n], dtype, bits=4)
    cache.append(k.to(TDT[dtype]), v.to(TDT[dtype]), [n], np.zeros(n, np.uint8))
    scale = 1 / math.sqrt(d)
    got = cache.decode_attention_layers(q, scale)
    # the one row's logit is 40, with magnitudes that are added of some eight times that
    close_groups(got[:, 0], expected(cache, 0, q, n, scale), deviation=40.0)
    assert cache.device_status() == 0


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("size", [1e33, 4e36, 3e37])
@pytest.mark.parametrize("n,segments", [(1024, ONE), (1024, MANY), (20011, ONE)])
def test_values_near_the_largest(d, size, n, segments):
    """Outputs far below the largest 32-bit number, times weights that are not."""
    if n > 2000 and d in (80, 96):
        pytest.skip("the longer sequence at the least and the greatest width")
    decode(torch.full((n, groups(d)), size), d, "bf16", segments, deviation=max(1.0, math.sqrt(n / 1000)))


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("sign", [1, -1])
def test_queries_near_the_largest(d, sign):
    """Columns whose sum is past the largest 32-bit number; the logits are not."""
    n, H = 500, 2
    g = torch.Generator(device="cuda")
    g.manual_seed(13)
    k, v = (torch.empty(1, n, H, d, device="cuda").normal_(generator=g).bfloat16() for _ in range(2))
    cache = kvc.KVCache(1, H, d, [n], "bf16", bits=4)
    cache.append(k, v, [n], np.zeros(n, np.uint8))
    q = torch.full((1, 1, H, d), sign * 2e37, dtype=torch.bfloat16, device="cuda")
    scale = float(np.float32(1.6e-37 / d))
    got = cache.decode_attention_layers(q, scale)
    # a group's sum of the query is 32 columns of 3.2 / d each, where usual ones leave sqrt(32 / d)
    close_groups(got[:, 0], expected(cache, 0, q, n, scale), deviation=32 * 3.2 / d / math.sqrt(32 / d))
    assert cache.device_status() == 0


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("size,q_size", [(3e36, 1.0), (1e37, 1e-2), (1e30, 1e-5)])
def test_large_keys_and_a_small_scale(d, size, q_size):
    n, H = 500, 2
    g = torch.Generator(device="cuda")
    g.manual_seed(14)
    k, v = (torch.empty(1, n, H, d, device="cuda").normal_(generator=g) for _ in range(2))
    cache = kvc.KVCache(1, H, d, [n], "bf16", bits=4)
    cache.append((k * size).bfloat16(), v.bfloat16(), [n], np.zeros(n, np.uint8))
    q = (torch.empty(1, 1, H, d, device="cuda").normal_(generator=g) * q_size).bfloat16()
    scale = float(np.float32(1 / math.sqrt(d) / size / q_size))
    got = cache.decode_attention_layers(q, scale)
    close_groups(got[:, 0], expected(cache, 0, q, n, scale))
    assert cache.device_status() == 0
