"""The learner-side operators where the server, the learner and others work on streams of their own."""
import pytest

pytestmark = pytest.mark.gpu

LONG = 200_000_000     # cycles of a kernel that only waits: a tenth of a second


def _server(n, stream=None):
    import torch
    from paper_1509_04210_b200 import binding as rb
    ps = rb.ParameterServer(n, 1, 1, 0.1, stream=stream)
    theta = torch.randn(n, device="cuda", generator=torch.Generator("cuda").manual_seed(n)) * 0.01
    torch.cuda.synchronize()
    return ps, theta


@pytest.mark.parametrize("transpose", [False, True])
def test_a_pull_waits_for_the_learners_stream_and_the_learners_stream_for_it(transpose):
    # the server on the legacy stream, the learner on one of torch's, which that does not wait for
    import torch
    from paper_1509_04210_b200 import learner as L
    rows, cols = 520, 1000
    ps, theta = _server(rows * cols)
    ps.set_weights(theta)
    ps.sync()
    held = theta.view(rows, cols)
    want = L.mx4_dequantize(L.mx4_quantize(held, transpose))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    reused = []
    with torch.cuda.stream(side):
        for _ in range(4):
            # a buffer that a long line of work on the learner's stream still reads when it is given back
            old = L.mx4_quantize(torch.full_like(held, 3.0), transpose)
            ptr = old.codes_ptr
            torch.cuda._sleep(LONG)
            seen = L.mx4_dequantize(old)
            del old
            q, ts = L.pull_mx4(ps, 0, rows, cols, transpose)
            got = L.mx4_dequantize(q)                       # at once, with no wait on the host
            reused.append(q.codes_ptr == ptr)
            assert ts == 0 and bool((seen == 3.0).all()) and torch.equal(got, want)
            # and into a matrix that earlier work reads
            torch.cuda._sleep(LONG)
            before = L.mx4_dequantize(q)
            L.mx4_quantize(torch.full_like(held, -2.0), transpose, out=q)
            torch.cuda._sleep(LONG)
            other = L.mx4_dequantize(q)
            L.pull_mx4(ps, 0, rows, cols, transpose, out=q)
            assert torch.equal(L.mx4_dequantize(q), want)
            assert torch.equal(before, want) and bool((other == -2.0).all())
            del q, got, seen
    assert any(reused)                                      # the case this is about: the allocator gives the same memory
    ps.close()


def test_a_pull_from_a_busy_server_is_used_at_once():
    import torch
    from paper_1509_04210_b200 import learner as L
    rows, cols = 300, 640
    theirs = torch.cuda.Stream()
    ps, theta = _server(rows * cols, theirs)
    want = L.mx4_dequantize(L.mx4_quantize(theta.view(rows, cols)))
    torch.cuda.synchronize()
    with torch.cuda.stream(theirs):
        torch.cuda._sleep(LONG)
    ps.set_weights(theta)                                   # behind that, on the server's stream
    q, _ = L.pull_mx4(ps, 0, rows, cols)
    assert torch.equal(L.mx4_dequantize(q), want)
    y = L.mx4_matmul(theta.view(rows, cols)[:3], q, torch.float32)
    again = L.mx4_matmul(theta.view(rows, cols)[:3], L.mx4_quantize(theta.view(rows, cols)), torch.float32)
    assert torch.equal(y, again)
    # a pull that is dropped: what its memory is used for next is not written over
    with torch.cuda.stream(theirs):
        torch.cuda._sleep(LONG)
    x = torch.full((rows, cols), 1.5, device="cuda")
    q, _ = L.pull_mx4(ps, 0, rows, cols)
    ptr = q.codes_ptr
    del q
    taken = []
    while not any(t.codes_ptr == ptr for t in taken) and len(taken) < 100:      # until that memory is given out again
        taken.append(L.mx4_quantize(x))
    torch.cuda.synchronize()
    assert taken[-1].codes_ptr == ptr and all(bool((L.mx4_dequantize(t) == 1.5).all()) for t in taken)
    ps.close()


def test_pulls_on_another_stream_can_be_captured():
    import torch
    from paper_1509_04210_b200 import learner as L
    rows, cols = 64, 96
    theirs = torch.cuda.Stream()
    ps, theta = _server(rows * cols, theirs)
    ps.set_weights(theta)
    ps.sync()
    q, _ = L.pull_mx4(ps, 0, rows, cols)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.pull_mx4(ps, 0, rows, cols, out=q)
        got = L.mx4_dequantize(q)
    ps.set_weights(theta * 2.0)
    ps.sync()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, L.mx4_dequantize(L.mx4_quantize(theta.view(rows, cols) * 2.0)))
    ps.close()


def test_a_pull_may_be_torchs_first_use_of_the_gpu():
    import os
    import subprocess
    import sys

    program = """
import numpy as np
from paper_1509_04210_b200 import binding as rb, learner as L
ps = rb.ParameterServer(64 * 96, 1, 1, 0.1)
ps.set_weights_host(np.full(64 * 96, 1.5, dtype=np.float32))
q, ts = L.pull_mx4(ps, 0, 64, 96)
import torch
assert ts == 0 and bool((L.mx4_dequantize(q, torch.float32) == 1.5).all()) and q.codes.shape == (64, 48)
L.sync()
ps.close()
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", program], cwd=root, check=True, timeout=120)
