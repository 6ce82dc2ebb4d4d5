"""What copies between caches of 16 and 4 bits make of rotated keys, and of a source that ends."""
import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc
from _packed import stored
from _serving import TDT, collected  # noqa: F401

pytestmark = pytest.mark.gpu


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
