"""Memory that a cache's calls use belongs to torch's pool: what a stream still uses is not given out again, and what the
pool had from a stream's work is not used before that work is complete."""
import types

import numpy as np
import pytest
import torch

import paper_2310_08152_gb300 as kvc

HERE, SIDE, DEFAULT = 1, 2, 0  # the current stream's handle, another's and the default stream's


class Pool:
    """Stands in for torch.cuda and what it allocates; `log` lists what happens in order."""

    def __init__(self, monkeypatch):
        self.log, self.capturing, self.made = [], set(), 0
        pool = self

        class Tensor:
            device = "cuda:0"

            def __init__(self, n):
                self.n, self.id, pool.made = n, pool.made, pool.made + 1
                pool.log.append(("made", self.id))

            def numel(self):
                return self.n

            def element_size(self):
                return 1

            def data_ptr(self):
                return 256 * (1 + self.id)

            def record_stream(self, stream):
                pool.log.append(("told", self.id, stream.cuda_stream))

            def __del__(self):
                pool.log.append(("dropped", self.id))

        class Event:
            def record(self):
                pool.log.append(("marked",))

            def synchronize(self):
                pool.log.append(("host waits",))

        class Stream:
            def __init__(self, handle, device=None):
                self.cuda_stream = handle or 1000  # as torch does: a new stream where the handle is 0

            def wait_event(self, event):
                pool.log.append(("waits", self.cuda_stream))

        class current:
            at = HERE

            def __init__(self, stream):
                self.new = stream.cuda_stream

            def __enter__(self):
                self.old, current.at = current.at, self.new

            def __exit__(self, *exc):
                current.at = self.old

        self.current = current
        default = Stream(1)
        default.cuda_stream = DEFAULT
        cuda = types.SimpleNamespace(Event=Event, ExternalStream=Stream, stream=current, synchronize=lambda d=None: None,
                                     default_stream=lambda device=None: default,
                                     current_device=lambda: 0, is_current_stream_capturing=lambda: current.at in pool.capturing)
        monkeypatch.setattr(torch, "cuda", cuda)
        monkeypatch.setattr(torch, "empty", lambda n, **kw: Tensor(n))
        monkeypatch.setattr(torch, "zeros", lambda *shape, **kw: Tensor(int(np.prod(shape))))
        monkeypatch.setattr(kvc, "_stream_handle", lambda s: current.at if s is None else s if isinstance(s, int) else s.cuda_stream)
        monkeypatch.setattr(kvc, "_dev", lambda t, *a, **kw: t)
        for name in ("kvc_set_prefix", "kvc_decode_attention_shared", "kvc_set_scores", "kvc_decode_attention_scored",
                     "kvc_score_prompt", "kvc_compress_spans"):
            monkeypatch.setattr(kvc, name, lambda *a, _name=name, **kw: pool.log.append((_name,)))
        monkeypatch.setattr(kvc, "kvc_prefix_scratch_bytes", lambda h: 4096)
        monkeypatch.setattr(kvc, "kvc_score_scratch_bytes", lambda h, n_q: 64 * int(np.sum(n_q)))
        lib = types.SimpleNamespace(kvc_thread_capture_mode=lambda mode: pool.log.append(("mode", mode)) or 0,
                                    kvc_evict=lambda *a: pool.log.append(("kvc_evict",)) or 0)
        monkeypatch.setattr(kvc, "lib", lambda: lib)

    def cache(self, b=2):
        c = object.__new__(kvc.KVCache)
        budget = np.zeros((2, b), np.int64)
        c.__dict__.update(M=3, H=4, d=64, b=b, C=10, torch_dtype=torch.float16, handle=None, scores=None, _scores=None, prefix=None,
                          _prefix_scratch=None, _score_scratch=None, _score_counts=None, _budget=budget,
                          _budget_at=budget.ctypes.data, k=types.SimpleNamespace(device="cuda:0"))
        return c

    def before(self, *events):
        """Each of the events is in the log, in this order."""
        at = [self.log.index(e) for e in events]
        assert at == sorted(at), (events, self.log)


@pytest.fixture
def pool(monkeypatch):
    return Pool(monkeypatch)


@pytest.fixture
def prefix():
    return types.SimpleNamespace(handle=7)


def test_prefix_scratch(pool, prefix):
    c = pool.cache()
    c.set_prefix(prefix, [0, 0])
    c.decode_attention_shared(None, 1.0, out=object(), stream=SIDE)
    c.set_prefix(None)
    pool.before(("made", 0), ("waits", SIDE), ("kvc_decode_attention_shared",), ("dropped", 0))
    pool.before(("told", 0, SIDE), ("dropped", 0))


def test_prefix_scratch_that_is_replaced(pool, prefix):
    c = pool.cache()
    c.set_prefix(prefix, [0, 0])
    with pool.current(types.SimpleNamespace(cuda_stream=SIDE)):  # by torch's current stream
        c.decode_attention_shared(None, 1.0, out=object())
    c.set_prefix(prefix, [1, 1])
    pool.before(("waits", SIDE), ("kvc_decode_attention_shared",), ("dropped", 0))
    pool.before(("told", 0, SIDE), ("dropped", 0))
    c.decode_attention_shared(None, 1.0, out=object())  # where it was made: nothing to order
    assert not [e for e in pool.log if e[0] == "told" and e[1] == 1]


def test_score_scratch(pool):
    """A call on a stream, and a larger one that names none."""
    c = pool.cache()
    c.score_prompt(0, None, [3, 4], 1.0, stream=SIDE)
    pool.before(("made", 0), ("waits", SIDE), ("kvc_score_prompt",))
    c.score_prompt(0, None, [30, 40], 1.0)
    pool.before(("told", 0, SIDE), ("dropped", 0))


@pytest.mark.parametrize("call", ["scored", "prompt", "evict", "compress"])
def test_scores_that_are_replaced(pool, call):
    c = pool.cache()
    c.attach_scores()
    if call == "scored":
        c.decode_attention_scored(None, 1.0, out=object(), stream=SIDE)
    elif call == "prompt":
        c.score_prompt(0, None, [3, 4], 1.0, stream=SIDE)
    elif call == "evict":
        c.evict(5, 2, stream=SIDE)
    else:
        c.compress_spans([0], [1], [2], stream=SIDE)
    c.attach_scores()
    pool.before(("told", 0, SIDE), ("dropped", 0))
    pool.before(("waits", SIDE), ("told", 0, SIDE))


def test_the_default_stream_is_one_too(pool, prefix):
    c = pool.cache()
    c.set_prefix(prefix, [0, 0])
    c.decode_attention_shared(None, 1.0, out=object(), stream=DEFAULT)
    c.set_prefix(None)
    pool.before(("waits", DEFAULT), ("told", 0, DEFAULT), ("dropped", 0))


def test_stream_is_ordered_once(pool, prefix):
    c = pool.cache()
    c.set_prefix(prefix, [0, 0])
    for _ in range(3):
        c.decode_attention_shared(None, 1.0, out=object(), stream=SIDE)
    assert pool.log.count(("waits", SIDE)) == pool.log.count(("told", 0, SIDE)) == 1


def test_first_use_in_a_capture(pool, prefix):
    """A stream that is being captured takes in no wait for work outside: the host does, with the thread's capture mode
    relaxed for it."""
    c = pool.cache()
    c.set_prefix(prefix, [0, 0])
    pool.capturing = {SIDE}
    c.decode_attention_shared(None, 1.0, out=object(), stream=SIDE)
    pool.before(("mode", 2), ("host waits",), ("mode", 0), ("kvc_decode_attention_shared",))
    assert ("waits", SIDE) not in pool.log


# ------------------------------------------------------------------------------------------
# on a GPU
# ------------------------------------------------------------------------------------------

def _samples(n=8, rows=900):
    from _serving import make, query

    prefix, _ = make(2, 8, 64, [rows], seed=1)
    own, g = make(2, 8, 64, [3] * n, seed=2, pos=np.concatenate([rows + np.arange(3)] * n).astype(np.int32))
    return prefix, own, query(own, g)


@pytest.mark.gpu
@pytest.mark.parametrize("again", [False, True])
def test_prefix_dropped_behind_a_decode_on_another_stream(again):
    prefix, own, q = _samples()
    own.set_prefix(prefix, [0] * 8)
    ref = own.decode_attention_shared(q, 0.125)
    side, out = torch.cuda.Stream(), torch.empty_like(ref)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)  # the decode is queued behind some 10 ms
    own.decode_attention_shared(q, 0.125, out=out, stream=side)
    own.set_prefix(prefix if again else None, [0] * 8)
    # what the pool gives out now is written on the current stream at once
    taken = [torch.full((kvc.kvc_prefix_scratch_bytes(own.handle),), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(out, ref) and all(bool((t == 255).all()) for t in taken)
    assert own.device_status() == 0


@pytest.mark.gpu
def test_prefix_made_and_dropped_on_another_stream_than_the_decode_s():
    """Made on a side stream, used on the default one, dropped and its memory given out again on the side stream."""
    prefix, own, q = _samples()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        own.set_prefix(prefix, [0] * 8)
    ref = own.decode_attention_shared(q, 0.125)
    out = torch.empty_like(ref)
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    own.decode_attention_shared(q, 0.125, out=out)
    own.set_prefix(None)
    n = kvc.kvc_prefix_scratch_bytes(own.handle)
    with torch.cuda.stream(side):
        taken = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(out, ref) and all(bool((t == 255).all()) for t in taken)
    assert own.device_status() == 0


@pytest.mark.gpu
def test_scratch_is_made_behind_work_of_its_own_stream():
    """The pool gives a block that work queued on the current stream still writes; the call runs on another stream."""
    prefix, own, q = _samples()
    own.set_prefix(prefix, [0] * 8)
    ref = own.decode_attention_shared(q, 0.125)
    own.set_prefix(None)
    torch.cuda.synchronize()
    side, out = torch.cuda.Stream(), torch.empty_like(ref)
    n = kvc.kvc_prefix_scratch_bytes(own.handle)
    torch.cuda._sleep(20_000_000)
    busy = [torch.full((n,), 1, dtype=torch.uint8, device="cuda") for _ in range(2)]
    del busy
    own.set_prefix(prefix, [0] * 8)
    own.decode_attention_shared(q, 0.125, out=out, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, ref)
    assert own.device_status() == 0


@pytest.mark.gpu
def test_score_scratch_grows_behind_a_call_on_another_stream():
    from _serving import make

    cache, g = make(1, 4, 64, [600], seed=3)
    q = torch.empty(600, 4, 64, dtype=torch.float16, device="cuda").normal_(generator=g)
    cache.attach_scores()
    cache.score_prompt(0, q[-100:], [100], 0.125)
    cache.score_prompt(0, q, [600], 0.125)
    ref = cache.scores.clone()
    other, _ = make(1, 4, 64, [600], seed=3)
    other.attach_scores()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    other.score_prompt(0, q[-100:], [100], 0.125, stream=side)
    done = torch.cuda.Event()
    done.record(side)
    need = kvc.kvc_score_scratch_bytes(other.handle, [100])
    torch.cuda.current_stream().wait_event(done)
    other.score_prompt(0, q, [600], 0.125)
    taken = torch.full((max(need, 256),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(other.scores, ref) and bool((taken == 255).all())
    assert cache.device_status() == 0 and other.device_status() == 0


@pytest.mark.gpu
def test_shared_decode_in_a_graph():
    prefix, own, q = _samples()
    own.set_prefix(prefix, [0] * 8)
    ref = own.decode_attention_shared(q, 0.125)
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(ref)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        own.decode_attention_shared(q, 0.125, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
    assert own.device_status() == 0


@pytest.mark.gpu
def test_a_plan_is_not_uploaded_in_a_capture():
    """The shared decode and the prompt scores refuse a capture whose plan is not on the device yet; the capture goes on."""
    prefix, own, q = _samples()
    own.set_prefix(prefix, [0] * 8)
    ref = own.decode_attention_shared(q, 0.125)
    one = own.decode_attention_shared(q[:1].contiguous(), 0.125, n_layers=1)
    torch.cuda.synchronize()
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(one)
    part, all_out = q[:1].contiguous(), torch.zeros_like(ref)
    prefix.attach_scores()
    window = torch.zeros(9, 8, 64, dtype=torch.float16, device="cuda")
    prefix.score_prompt(0, window, [9], 0.125)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        own.decode_attention_shared(part, 0.125, out=out, n_layers=1)
        with pytest.raises(kvc.KvcError) as e:  # a plan for another number of layers
            own.decode_attention_shared(q, 0.125, out=all_out)
        assert e.value.status == 5
        with pytest.raises(kvc.KvcError) as e:  # other queries
            prefix.score_prompt(0, window[:8], [8], 0.125)
        assert e.value.status == 5
        prefix.score_prompt(0, window, [9], 0.125)
    before = prefix.scores.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, one) and torch.all(all_out == 0)
    assert abs(float((prefix.scores - before).double().sum()) - 9 * 8) <= 1e-3
    assert torch.equal(own.decode_attention_shared(q, 0.125), ref)
    assert own.device_status() == 0 and prefix.device_status() == 0
