"""The example that runs the bounded cache's operators together, at a small size, against a plain record of its rows."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc

from _serving import attend, close, collected, rotate, rows_of  # noqa: F401

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("samples_of_a_prompt", os.path.join(ROOT, "examples", "samples_of_a_prompt.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype,rot,samples", [("f16", 64, 8), ("bf16", 0, 40)])
def test_prompt_to_samples(dtype, rot, samples):
    ex = example()
    cache = kvc.KVCache(2, 3, 64, [700], dtype, rotary_dim=rot)
    cache.attach_scores()
    kinds = ex.span_kinds(640)
    ex.ingest(cache, ex.Activations(cache, 1), kinds, 128, 150, 40, 0.125)
    assert cache.lengths()[0][0] == 150
    # every query's weights have gone to rows of its time; those of rows that went are gone
    total = float(cache.scores.double().sum())
    assert 0 < total <= 2 * 3 * 640 * (1 + 1e-5)
    first = int((kinds == kvc.NORMAL).sum())
    out = ex.sample(cache, samples, 5, first, 0.125, 7)
    # the same activations again, their last step's attention in 64 bits
    own = kvc.KVCache(2, 3, 64, [5] * samples, dtype, rotary_dim=rot)
    model = ex.Activations(own, 7)
    for t in range(5):
        k, v = model(2, samples), model(2, samples)
        own.append(k, v, np.ones(samples, np.int32), np.zeros(samples, np.uint8), pos=np.full(samples, first + t, np.int32))
        q = model(2, samples, sd=2.0)
    kp, vp = rows_of(cache, 0, 150)
    for s in range(samples):
        ko, vo = rows_of(own, s, 5)
        for m in range(2):
            ref, _ = attend(rotate(q[m, s], first + 4, rot), torch.cat([kp[m], ko[m]], 1), torch.cat([vp[m], vo[m]], 1),
                            list(range(155)), 0.125)
            close(out[m, s], ref, f"sample {s}, layer {m}")
    ex.go_on(cache, 6, 150, 40, 0.125, 3)
    assert cache.lengths()[0][0] == 150 and cache.device_status() == 0


def test_command():
    rows = example().main(["--layers", "2", "--heads", "4", "--d-head", "64", "--rotary", "0", "--prompt", "400", "--block", "128",
                           "--budget", "100", "--recent", "30", "--samples", "3", "--steps", "6"])
    assert rows == 100
