"""Shared prefixes and scores, as far as the library checks them before any device work."""
import numpy as np
import pytest

import paper_2310_08152_gb300 as kvc


def cache(b=2, M=1, H=8, d=64):
    """A cache's handle with buffers that nothing touches."""
    cfg, _ = kvc.make_config(M, H, d, [16] * b, "f16", 0, 10000.0, kvc.POLICY_PAPER, 0.0)
    cfg.k_base = cfg.v_base = cfg.pos_base = cfg.orig_base = cfg.workspace = 1 << 40
    cfg.workspace_bytes = 1 << 40
    return kvc.kvc_create(cfg)


class Scratch:
    """So much memory at an address."""

    def __init__(self, n):
        self.n = n

    def numel(self):
        return self.n

    def element_size(self):
        return 1

    def data_ptr(self):
        return 1 << 41


def set_prefix(c, prefix):
    kvc.kvc_set_prefix(c, prefix, [0, 1], Scratch(kvc.kvc_prefix_scratch_bytes(c)))


def test_prefixes_do_not_nest():
    a, b, c = cache(), cache(), cache()
    set_prefix(b, c)
    with pytest.raises(kvc.KvcError) as e:
        set_prefix(a, b)
    assert e.value.status == 2
    kvc.kvc_set_prefix(b, None, None, None)
    set_prefix(a, b)
    for h in (a, b, c):
        kvc.kvc_destroy(h)


@pytest.mark.gpu
def test_a_prefix_that_gets_one_later():
    from _serving import make, query

    (a, g), (b, _), (c, _) = (make(1, 2, 64, [5, 5], seed=i) for i in range(3))
    q = query(a, g)
    a.set_prefix(b, [0, 1])
    ref = a.decode_attention_shared(q, 0.125)
    b.set_prefix(c, [0, 1])
    with pytest.raises(kvc.KvcError) as e:
        a.decode_attention_shared(q, 0.125)
    assert e.value.status == 2
    b.set_prefix(None)
    assert np.array_equal(a.decode_attention_shared(q, 0.125).cpu(), ref.cpu())


def test_decodes_of_no_layers_do_nothing():
    """As the plain decode's, before anything else is looked at."""
    h = cache(M=2)
    lib, scale = kvc.lib(), 0.125
    for call in (lib.kvc_decode_attention_layers, lib.kvc_decode_attention_scored, lib.kvc_decode_attention_shared):
        for first in (0, 1, 2):
            assert call(h, first, 0, None, 0, scale, None, 0, None) == 0
        for first, n in ((0, -1), (-1, 0), (-1, 1), (3, 0), (1, 2)):
            assert call(h, first, n, None, 0, scale, None, 0, None) == 1
    kvc.kvc_destroy(h)


@pytest.mark.parametrize("b,M,H,d,most", [(2, 1, 8, 64, 1 << 19), (8, 1, 32, 128, 4 << 20), (64, 2, 32, 128, 27 << 20)])
def test_scratch_is_of_the_batch_s_size(b, M, H, d, most):
    """640 runs that splitting adds, of min(b, 128) queries each with d + 4 floats, besides M H b parts and the plan."""
    h = cache(b, M, H, d)
    n = kvc.kvc_prefix_scratch_bytes(h)
    kvc.kvc_destroy(h)
    parts = M * H * b + 640 * min(b, 128)
    assert parts * 4 * (d + 4) <= n <= min(most, parts * 4 * (d + 4) + 32 * (640 + b) + 12 * b + 1024)


@pytest.mark.gpu
@pytest.mark.parametrize("members,n", [(1, 200000), (2, 150000), (17, 60000), (33, 60000), (129, 30000)])
@pytest.mark.parametrize("M,H", [(1, 1), (1, 7)])
def test_plans_fit_the_scratch(members, n, M, H):
    """Few heads and a long prefix: as many runs as there may be; what lies behind the scratch is left alone."""
    import torch

    from _serving import query
    from test_gpu_shared_prefix import check, pair

    parent, own = [0] * members, [1] * members
    prefix, c, g = pair(M, H, 64, [n], parent, own, seed=members)
    need = kvc.kvc_prefix_scratch_bytes(c.handle)
    memory = torch.full((need + 65536,), 77, dtype=torch.uint8, device="cuda")
    kvc.kvc_set_prefix(c.handle, prefix.handle, parent, memory[:need])
    q = query(c, g)
    out = c.decode_attention_shared(q, 0.125)
    check(prefix, c, parent, own, q, 0.125, out)
    assert bool((memory[need:] == 77).all())
    kvc.kvc_set_prefix(c.handle, None, None, None)
