"""Kernels that let the next one start before they end, by their source: whether it reads too early shows only where launches
are queued without a gap, and then as a read or write out of range.

A kernel's wait covers the kernel before it, not the ones before that.  So a kernel that reads ahead of its wait, because the one
before it was a decode, relies on that decode: it lets the next kernel start when what it had to wait for itself is complete."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_08152_gb300", "csrc")


def _source(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"\s+", " ", re.sub(r"//[^\n]*", "", text))


def _kernel(src, name):
    """The body of a kernel."""
    at = src.index("{", src.index(name + "("))
    depth = 0
    for i in range(at, len(src)):
        depth += (src[i] == "{") - (src[i] == "}")
        if depth == 0:
            return src[at:i + 1]


def _trigger_allowed(body):
    """Whether every pdl_launch_dependents() of a kernel that may read ahead of its wait stands behind that wait, or where
    kv_before_wait says that nothing is to be waited for."""
    calls = [m.start() for m in re.finditer(r"pdl_launch_dependents\(\);", body)]
    return bool(calls) and all(re.search(r"(pdl_wait\(\); |if \(p\.kv_before_wait\) )$", body[:at]) for at in calls)


def test_the_check_sees_a_trigger_that_comes_first():
    assert not _trigger_allowed("{ pdl_launch_dependents(); if (!p.kv_before_wait) pdl_wait(); f(); }")
    assert _trigger_allowed("{ if (p.kv_before_wait) pdl_launch_dependents(); if (!p.kv_before_wait) { pdl_wait(); pdl_launch_dependents(); } }")


def test_packed_decode_lets_the_next_start_behind_what_it_waits_for():
    body = _kernel(_source("packed_decode.cu"), "packed_decode_kernel")
    assert _trigger_allowed(body)
    # and it reads state, rows and the plan behind its wait where the kernel before it was not a decode
    wait = body.index("pdl_wait();")
    assert body[:wait].endswith("if (!p.kv_before_wait) { ")
    assert not re.search(r"p\.(P|ds|q|parts|counters)\b|bulk_g2s", body[:wait])


def test_kernels_ahead_of_a_16_bit_decode_do_not_let_it_start():
    """Its kernels read the plan ahead of their wait and let the next one start at once, which is in order as long as what writes
    a 16-bit cache's rows and state does not do the like; a cut waits before anything else."""
    for name in ("kernels.cu", "copy.cu", "evict.cu"):
        src = _source(name)
        for kernel in re.findall(r"__global__ void (?:__launch_bounds__\([^)]*\) )?(\w+)\(", src):
            body = _kernel(src, kernel)
            if "pdl_launch_dependents" in body:
                assert kernel in ("compact_scan_kernel", "decode_kernel", "decode_cta_kernel"), kernel
    move = _kernel(_source("kernels.cu"), "compact_move_kernel")
    assert "pdl_wait();" in move
    assert re.match(r"\{ pdl_wait\(\);", _kernel(_source("copy.cu"), "drop_image_kernel"))
