"""What copies between caches of 16 and 4 bits make of rows at the types' ends, of rotated keys, and of a source that ends."""
import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc
from _packed import stored, unpack16, values
from _serving import TDT, collected, rows_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 80, 96, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_finite_rows_come_back_finite(d, dtype):
    """A step that is rounded up puts a group's greatest value past the type's largest, by half a step at most."""
    t = TDT[dtype]
    top = torch.finfo(t).max
    n, H = 300, 2
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.empty(1, n, H, d, device="cuda").normal_(generator=g).to(t)
    low = -1.0 if dtype == "f16" else -0.5  # in bf16 a range of 1.5 x 3.39e38, which binary32 does not hold: NaN by definition
    x[0, 0:40, :, 3], x[0, 0:40, :, 7] = top, 0.0
    x[0, 40:80, :, 33:64:2], x[0, 40:80, :, 34:64:2] = top, low * top
    x[0, 80:120] = top
    x[0, 120:160, :, ::3] = torch.linspace(0.3, 1.0, 40, device="cuda")[:, None, None].to(t) * top
    x[0, 160:200, :, 5] = -top
    x[0, 210:250, :, :32] = torch.linspace(0.0, 0.9, 40, device="cuda")[:, None, None].to(t) * top  # steps of all kinds
    x[0, 210:250, :, 3] = top
    x[0, 200, 0, 3] = float("nan")
    x[0, 201, 1, 40] = float("inf")
    cache = kvc.KVCache(1, H, d, [n], dtype, bits=4)
    cache.append(x, x, [n], np.zeros(n, np.uint8))
    held = values(*stored(cache, 0, n))[0]
    assert (held[torch.isfinite(held)].abs() > top).any()  # the case is there
    back = [y[0].cpu() for y in rows_of(unpack16(cache), 0, n)]
    want = held.clamp(max=top).to(t)  # a NaN stays one
    nans = 64 + (0 if dtype == "f16" else 40 * H * 32)  # two groups that are not finite, and 40 rows' of too large a range
    for y in back:
        nan = torch.isnan(want)
        assert torch.equal(torch.isnan(y), nan) and nan.sum() == nans
        assert torch.equal(y[~nan], want[~nan])
    # and a row that has been there and back stays within a step's rounding of itself
    again = kvc.KVCache(1, H, d, [n], dtype, bits=4)
    again.copy_from(unpack16(cache), [0], [0])
    rows = [i for i in range(n) if i not in (200, 201) and (dtype == "f16" or not 40 <= i < 80)]
    assert torch.isfinite(values(*stored(again, 0, n))[0][:, rows]).all()


@pytest.mark.parametrize("d,rot", [(64, 64), (64, 16), (80, 80), (80, 48), (96, 96), (128, 128), (128, 32)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_rotated_keys_are_those_of_the_16_bit_cache(d, rot, dtype):
    """An append to 4 bits and a copy of the 16-bit cache's rows give the same codes and pairs: of many tokens, of a token a
    sequence, and a layer at a time."""
    M, H, lens = 2, 3, [700, 90, 1]
    g = torch.Generator(device="cuda")
    g.manual_seed(d + rot)
    caches = [kvc.KVCache(M, H, d, [n + 8 for n in lens], dtype, rotary_dim=rot, bits=bits) for bits in (16, 4)]
    pos = np.concatenate([np.arange(700) * 37, 100000 + np.arange(90), [5]]).astype(np.int32)  # far positions among them

    def append(n_new, pos=None, by_layer=False):
        n = sum(n_new)
        x = [torch.empty(M, n, H, d, dtype=TDT[dtype], device="cuda").normal_(generator=g) for _ in range(2)]
        for c in caches:
            if by_layer:
                for m in range(M):
                    c.append(x[0][m].contiguous(), x[1][m].contiguous(), n_new, np.zeros(n, np.uint8), layer=m)
            else:
                c.append(*x, n_new, np.zeros(n, np.uint8), pos=pos)

    append(lens, pos)
    append([1, 1, 1])
    append([0, 2, 1], by_layer=True)
    wide, narrow = caches
    copy = kvc.KVCache(M, H, d, [n + 8 for n in lens], dtype, rotary_dim=rot, bits=4)
    copy.copy_from(wide, range(3), range(3))
    for s, n in enumerate(narrow.lengths()[0]):
        for which in "kv":
            for a, b, name in zip(stored(narrow, s, int(n), which), stored(copy, s, int(n), which), ("codes", "steps", "least values")):
                assert torch.equal(a, b), (s, which, name, int((a != b).sum()))


@pytest.mark.parametrize("bits", [(16, 4), (4, 16), (16, 16)])
def test_a_source_that_ends_while_its_copy_is_queued(bits):
    """On another stream: the source is dropped as soon as the call has returned, and what is made next may get its memory."""
    M, H, d, n = 8, 16, 64, 3000
    side = torch.cuda.Stream()

    def copied(drop):
        g = torch.Generator(device="cuda")
        g.manual_seed(1)
        x = [torch.empty(M, n, H, d, dtype=torch.float16, device="cuda").normal_(generator=g) for _ in range(2)]
        source = kvc.KVCache(M, H, d, [n], bits=bits[0])
        target = kvc.KVCache(M, H, d, [n], bits=bits[1])
        source.append(*x, [n], np.zeros(n, np.uint8))
        torch.cuda.synchronize()
        sizes = [t.numel() * t.element_size() for t in (source.k, source.v, source.pos, source.orig)]
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)  # some 10 ms
        target.copy_from(source, [0], [0], stream=side)
        if drop:
            del source
            over = [torch.zeros(m, dtype=torch.uint8, device="cuda") for m in sizes]
        torch.cuda.synchronize()
        return target.k.view(torch.uint8).clone(), target.v.view(torch.uint8).clone(), target.pos.clone(), target.orig.clone()

    for a, b in zip(copied(True), copied(False)):
        assert torch.equal(a, b)
