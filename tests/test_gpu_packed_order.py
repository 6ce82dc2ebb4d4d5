"""Calls on a cache of 4 bits whose kernels are queued behind each other without a gap, as on a GPU that is behind or in a graph:
they give what they give one by one, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc
from _serving import TDT

pytestmark = pytest.mark.gpu

KEEP_BUSY = 4_000_000  # clock cycles, about 2 ms: what is queued behind it runs without a gap


def run(calls, queued):
    """Makes the calls, on a GPU that is busy until all are queued or waited for one by one."""
    torch.cuda.synchronize()
    if queued:
        torch.cuda._sleep(KEEP_BUSY)
    for call in calls:
        call()
        if not queued:
            torch.cuda.synchronize()
    torch.cuda.synchronize()


def rows(g, M, n, H, d, dtype):
    return [torch.empty(M, n, H, d, dtype=TDT[dtype], device="cuda").normal_(generator=g) for _ in range(2)]


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (80, "bf16"), (96, "f16"), (128, "bf16")])
@pytest.mark.parametrize("lens", [[3000], [1, 2000, 62]])
def test_prompt_then_a_decode_of_each_layer(d, dtype, lens):
    """A new cache's prompt, whose append runs far longer than the decode's launches take, and the decode of one layer after
    the other; then a long block more, which crosses tiles."""
    M, H = 6, 2
    more = [900] * len(lens)

    def outputs(queued):
        g = torch.Generator(device="cuda")
        g.manual_seed(5)
        first, second = rows(g, M, sum(lens), H, d, dtype), rows(g, M, sum(more), H, d, dtype)
        q = torch.empty(M, len(lens), H, d, dtype=TDT[dtype], device="cuda").normal_(generator=g)
        cache = kvc.KVCache(M, H, d, [n + 900 for n in lens], dtype, rotary_dim=32, bits=4)
        out = torch.full((2, M, len(lens), H, d), 7.0, device="cuda")
        calls = []
        for i, (x, n) in enumerate(((first, lens), (second, more))):
            calls.append(lambda x=x, n=n: cache.append(*x, n, np.zeros(sum(n), np.uint8)))
            calls += [lambda i=i, m=m: cache.decode_attention(m, q[m], 0.1, out=out[i, m]) for m in range(M)]
        run(calls, queued)
        assert cache.device_status() == 0
        return out

    want = outputs(False)
    assert torch.isfinite(want).all() and not (want == 7.0).any()
    for _ in range(3):
        assert torch.equal(outputs(True), want)


@pytest.mark.parametrize("d", [64, 128])
def test_steps_of_one_layer_after_the_other(d):
    """A token a sequence over a tile's edge, and each layer's decode, step after step."""
    M, H, lens = 4, 2, [60, 124, 5]

    def outputs(queued):
        g = torch.Generator(device="cuda")
        g.manual_seed(6)
        x = rows(g, M, sum(lens), H, d, "f16")
        cache = kvc.KVCache(M, H, d, [n + 16 for n in lens], "f16", bits=4)
        cache.append(*x, lens, np.zeros(sum(lens), np.uint8))
        q = torch.empty(M, 3, H, d, dtype=torch.float16, device="cuda").normal_(generator=g)
        out = torch.empty(12, M, 3, H, d, device="cuda")
        calls = []
        for i in range(12):
            t = rows(g, M, 3, H, d, "f16")
            calls.append(lambda t=t: cache.append(*t, [1] * 3, np.zeros(3, np.uint8)))
            calls += [lambda i=i, m=m: cache.decode_attention(m, q[m], 0.1, out=out[i, m]) for m in range(M)]
        run(calls, queued)
        assert cache.device_status() == 0
        return out

    want = outputs(False)
    for _ in range(3):
        assert torch.equal(outputs(True), want)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f16")])
def test_captured_append_and_decodes(d, dtype):
    """A step as a graph: its append's upload is a kernel parameter, so a replay writes the same rows and state again."""
    M, H, lens = 4, 2, [64, 31, 200]
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    x, t = rows(g, M, sum(lens), H, d, dtype), rows(g, M, 3, H, d, dtype)
    q = torch.empty(M, 3, H, d, dtype=TDT[dtype], device="cuda").normal_(generator=g)
    out = torch.empty(M, 3, H, d, device="cuda")
    cache = kvc.KVCache(M, H, d, [n + 4 for n in lens], dtype, bits=4)
    cache.append(*x, lens, np.zeros(sum(lens), np.uint8))
    cache.decode_attention(0, q[0], 0.1, out=out[0])  # the kernel's first use sets it up
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.append(*t, [1] * 3, np.zeros(3, np.uint8))
        for m in range(M):
            cache.decode_attention(m, q[m], 0.1, out=out[m])
    for seed in range(3):  # other rows in the same place
        for y in t:
            y.normal_(generator=g)
        torch.cuda.synchronize()
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = torch.stack([cache.decode_attention(m, q[m], 0.1) for m in range(M)])
        assert torch.equal(got, want)
    other = kvc.KVCache(M, H, d, [n + 4 for n in lens], dtype, bits=4)  # the last replay's rows, appended
    other.append(*x, lens, np.zeros(sum(lens), np.uint8))
    other.append(*t, [1] * 3, np.zeros(3, np.uint8))
    assert torch.equal(torch.stack([other.decode_attention(m, q[m], 0.1) for m in range(M)]), got)
    assert cache.device_status() == 0
