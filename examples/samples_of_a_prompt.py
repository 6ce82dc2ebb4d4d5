"""Many samples of one prompt under a bounded cache, with synthetic activations.

The prompt goes in block by block: its keys and values are appended, every layer's masked attention is run, the block's
attention weights are added to the rows' scores, the closed sentinel spans are freed, and the cache is brought back to its
budget by evicting what was attended to least.  Then `samples` continuations are generated over the one prompt cache, whose
rows are stored and read once for all of them; a second generation goes on from the prompt itself, step by step within the
budget.

  python examples/samples_of_a_prompt.py --prompt 2000 --budget 512 --samples 8 --steps 32
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2310_08152_gb300 as kvc  # noqa: E402


class Activations:
    """Stands in for a model: normal queries, keys and values of the cache's shape."""

    def __init__(self, cache: kvc.KVCache, seed: int):
        self.cache = cache
        self.gen = torch.Generator(device=cache.k.device)
        self.gen.manual_seed(seed)

    def __call__(self, *shape, sd: float = 1.0):
        c = self.cache
        x = torch.empty(*shape, c.H, c.d, dtype=c.torch_dtype, device=c.k.device)
        return x.normal_(0.0, sd, generator=self.gen)


def span_kinds(n: int, every: int = 64, interior: int = 32) -> np.ndarray:
    """One sentinel span in each `every` tokens."""
    k = np.zeros(n, np.uint8)
    for a in range(7, n - interior - 1, every):
        k[a], k[a + interior + 1] = kvc.CL, kvc.CR
    return k


def ingest(cache: kvc.KVCache, model: Activations, kinds: np.ndarray, block: int, budget: int, recent: int, scale: float):
    """The prompt into a cache of one sequence, block by block, within the budget after each block."""
    for a in range(0, kinds.size, block):
        new = kinds[a:a + block]
        n = [new.size]
        cache.append(model(cache.M, new.size), model(cache.M, new.size), n, new)
        for layer in range(cache.M):
            q = model(new.size, sd=2.0)
            cache.prefill_attention(layer, q, n, scale)
            cache.score_prompt(layer, q, n, scale)
        closed = cache.pending_spans(0)
        if closed:
            cache.compress_spans([0] * len(closed), *map(list, zip(*closed)))
        so_far = kinds[:a + block]
        if (so_far == kvc.CL).sum() == (so_far == kvc.CR).sum():  # an open span has to stay among the recent rows
            cache.evict(budget, recent)


def sample(prompt: kvc.KVCache, samples: int, steps: int, first_position: int, scale: float, seed: int) -> torch.Tensor:
    """The last step's attention outputs [M, samples, H, d] of `samples` continuations of the prompt."""
    own = kvc.KVCache(prompt.M, prompt.H, prompt.d, [steps] * samples, prompt.dtype, rotary_dim=prompt.rotary_dim,
                      rope_base=prompt.rope_base)
    own.set_prefix(prompt, [0] * samples)
    model = Activations(own, seed)
    kinds, one = np.zeros(samples, np.uint8), np.ones(samples, np.int32)
    out = torch.empty(prompt.M, samples, prompt.H, prompt.d, device=prompt.k.device)
    for t in range(steps):
        pos = np.full(samples, first_position + t, np.int32)
        own.append(model(prompt.M, samples), model(prompt.M, samples), one, kinds, pos=pos)
        own.decode_attention_shared(model(prompt.M, samples, sd=2.0), scale, out=out)
    torch.cuda.synchronize()
    if own.device_status() or prompt.device_status():
        raise RuntimeError("a kernel reported an error")
    return out


def go_on(prompt: kvc.KVCache, steps: int, budget: int, recent: int, scale: float, seed: int) -> torch.Tensor:
    """Generation from the prompt's own cache, which stays at its budget."""
    model = Activations(prompt, seed)
    out = torch.empty(prompt.M, 1, prompt.H, prompt.d, device=prompt.k.device)
    for _ in range(steps):
        prompt.append(model(prompt.M, 1), model(prompt.M, 1), [1], [kvc.NORMAL])
        prompt.decode_attention_scored(model(prompt.M, 1, sd=2.0), scale, out=out)
        prompt.evict(budget, recent)
    torch.cuda.synchronize()
    return out


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=8)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--d-head", type=int, default=80)
    ap.add_argument("--rotary", type=int, default=80)
    ap.add_argument("--dtype", choices=("f16", "bf16"), default="f16")
    ap.add_argument("--prompt", type=int, default=2000)
    ap.add_argument("--block", type=int, default=512)
    ap.add_argument("--budget", type=int, default=512)
    ap.add_argument("--recent", type=int, default=96)
    ap.add_argument("--samples", type=int, default=8)
    ap.add_argument("--steps", type=int, default=32)
    a = ap.parse_args(argv)
    scale = a.d_head ** -0.5
    kinds = span_kinds(a.prompt)
    cache = kvc.KVCache(a.layers, a.heads, a.d_head, [a.budget + 2 * a.block + a.steps], a.dtype, rotary_dim=a.rotary)
    cache.attach_scores()
    ingest(cache, Activations(cache, 1), kinds, a.block, a.budget, a.recent, scale)
    rows = int(cache.lengths()[0][0])
    print(f"prompt: {a.prompt} tokens, {rows} rows a head left")
    first = int((kinds == kvc.NORMAL).sum())
    sample(cache, a.samples, min(4, a.steps), first, scale, 2)  # warm-up
    t = time.perf_counter()
    out = sample(cache, a.samples, a.steps, first, scale, 2)
    t = time.perf_counter() - t
    print(f"{a.samples} samples of it: {a.samples * a.steps / t:.0f} tokens/s of cache and attention, {a.layers} layers")
    out = go_on(cache, a.steps, a.budget, a.recent, scale, 3)
    print(f"generation from it: {int(cache.lengths()[0][0])} rows a head after {a.steps} steps, outputs of deviation "
          f"{float(out.std()):.3f}")
    return rows


if __name__ == "__main__":
    main()
