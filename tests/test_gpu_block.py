"""The 8-bit product, the norm and the clipping together, as a learner's residual block uses them: every call of the example
against 64 bits, captured and replayed graphs, streams, two threads."""
import importlib.util
import os
import threading

import numpy as np
import pytest

import block_reference as ref
import learner_reference as lref
from test_gpu_learner import EPS, _close, _learner, _np, _torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "learner_block.py")
    spec = importlib.util.spec_from_file_location("learner_block", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _values(q):
    """What a tensor, FP8 matrix or checkpoint stands for, in 64 bits."""
    torch, L = _torch(), _learner()
    if isinstance(q, L.FP8):
        return _np(L.fp8_dequantize(q, torch.float32))
    return _np(L.act8_values(q, torch.float32)) if isinstance(q, L.Act8) else _np(q)


class _Checked:
    """The learner module with its results checked, from what each call was given."""

    def __init__(self, L):
        self.L, self.calls = L, []

    def __getattr__(self, name):
        f = getattr(self.L, name)
        if name not in ("rms_norm", "rms_norm_backward", "fp8_matmul", "fp8_quantize", "act8_weight_grad", "clip_gradients"):
            return f

        def call(*a, **kw):
            given = [_values(v) if hasattr(v, "shape") or isinstance(v, (self.L.FP8, self.L.Act8)) else [_values(t) for t in v] if isinstance(v, list) else v for v in a]
            more = {k: _values(v) if hasattr(v, "shape") and k in ("residual", "dsum") else v for k, v in kw.items()}
            got = f(*a, **kw)
            getattr(self, "_" + name)(got, a, kw, given, more)
            self.calls.append(name)
            return got

        return call

    def _out(self, got):
        return 2.0 ** -8 if got.dtype == _torch().bfloat16 else 0.0

    def _rms_norm(self, got, a, kw, given, more):
        x, w = given
        s = x + more["residual"] if more.get("residual") is not None else x
        if len(got) == 3:
            s = _torch().from_numpy(s.astype(np.float32)).bfloat16().double().numpy()
            np.testing.assert_array_equal(_np(got[1]), s)
        y, tol = ref.norm(s, w, 1e-6), 40 * U
        top = np.repeat(np.abs(y).reshape(len(y), -1, 128).max(axis=2), 128, axis=1)
        _close(_values(got[0]), y, np.maximum(np.abs(y) * (1 + tol) / 16, top / 224 * (1 + 2 * tol) * 2.0 ** -10) + tol * np.abs(y))
        top = np.repeat(np.abs(y).reshape(len(y), -1, 32).max(axis=2), 32, axis=1)
        _close(_values(got[-1]), y, top / 127 * (1 + tol) + tol * top)

    def _rms_norm_backward(self, got, a, kw, given, more):
        ds, dw, size, size_w = ref.norm_backward(*given, 1e-6, more.get("dsum"))
        _close(_np(got[0]), ds, 100 * U * size + 2.0 ** -8 * np.abs(ds))
        _close(_np(got[1]), dw, (len(ds) + 65) * U * size_w)

    def _fp8_matmul(self, got, a, kw, given, more):
        x = given[0] if isinstance(a[0], self.L.FP8) else ref.fp8_values(given[0])
        want, size = x @ given[1].T, np.abs(x) @ np.abs(given[1]).T
        _close(_np(got), want, x.shape[1] * EPS * size + self._out(got) * np.abs(want))

    def _fp8_quantize(self, got, a, kw, given, more):
        np.testing.assert_array_equal(_values(got), ref.fp8_values(given[0].T if kw.get("transpose") else given[0], kw.get("square", False)))

    def _act8_weight_grad(self, got, a, kw, given, more):
        _close(_np(got), given[0].T @ given[1], len(given[0]) * EPS * (np.abs(given[0]).T @ np.abs(given[1])))

    def _clip_gradients(self, got, a, kw, given, more):
        n, want = ref.clip(given[0], a[1])
        assert abs(got.item() - n) <= 6 * U * n
        for g, w in zip(a[0], want):
            _close(_np(g), w, 8 * U * np.abs(w))


def test_a_learners_step_call_by_call(monkeypatch):
    torch = _torch()
    ex = _example()
    from paper_1509_04210_b200 import binding as rb
    net = ex.Network(256, 384, 40, 2)
    ps = rb.ParameterServer(net.nparams, 1, 1, 0.1, stream=torch.cuda.current_stream())
    theta = net.initial(3)
    ps.set_weights(theta)
    l = ex.Learner(net, 5)
    checked = _Checked(ex.ln)
    monkeypatch.setattr(ex, "ln", checked)
    l.pull(ps)
    for k, v in net.views(theta).items():
        if k[0] != "norm":
            np.testing.assert_array_equal(_values(l.weights[k]), ref.fp8_values(_np(v), True))
            np.testing.assert_array_equal(_values(l.turned[k]), ref.fp8_values(_np(v), True).T)
    x = torch.randn(100, 256, device="cuda").bfloat16()
    loss = l.compute(x, torch.randint(0, 40, (100,), device="cuda"))
    before = _np(l.pushed)
    l.clip(0.5 * float(np.linalg.norm(before)))
    assert np.isfinite(loss.item()) and np.isfinite(before).all() and (before != 0).mean() > 0.9
    assert checked.calls.count("rms_norm") == checked.calls.count("rms_norm_backward") == 3 and checked.calls.count("fp8_matmul") == 12
    ps.push(l.pushed, l.ts)
    assert ps.step() == 1
    got = torch.empty(net.nparams, device="cuda")
    assert ps.pull(got) == 1
    _close(_np(got), _np(theta) - 0.1 * _np(l.pushed), 4 * U * (np.abs(_np(theta)) + np.abs(_np(l.pushed))))
    ps.close()


def test_the_example_runs():
    losses = _example().train(updates=6, learners=2, n=1, batch=64, width=128, hidden=256, classes=10, blocks=1)
    assert len(losses) >= 6 and np.isfinite(losses).all()


def _step(L, x, r, w, q, turned, grads, parts):
    """One block forward and backward and the clipping, on whatever stream is current."""
    torch = _torch()
    y, s, kept = L.rms_norm(x, w, r, fp8=True, keep=True)
    h = L.fp8_matmul(y, q)
    dh, saved = L.act8_forward("gelu", h)
    L.act8_weight_grad(dh, kept, out=grads[0])
    dy = L.fp8_matmul(dh, turned)
    ds, _ = L.rms_norm_backward(dy, s, w, dsum=r, out_weight=grads[1])
    norm = L.clip_gradients(grads, 0.25, out=parts)
    return [L.fp8_dequantize(y, torch.float32), s, h, dy, ds, norm] + list(parts) + [g.clone() for g in grads]


def _state(t, c, n, seed):
    torch, L = _torch(), _learner()
    gen = torch.Generator("cuda").manual_seed(seed)
    x, r = (torch.randn(t, c, device="cuda", generator=gen).bfloat16() for _ in range(2))
    w, m = torch.rand(c, device="cuda", generator=gen) + 0.5, torch.randn(n, c, device="cuda", generator=gen) * 0.05
    grads = [torch.zeros(n, c, device="cuda"), torch.zeros(c, device="cuda")]
    vector = torch.zeros(n * c + c, device="cuda", dtype=torch.bfloat16)
    parts = [vector[:n * c], vector[n * c:]]
    return [x, r, w, L.fp8_quantize(m, square=True), L.fp8_quantize(m, transpose=True, square=True), grads, parts]


@pytest.mark.parametrize("t,c,n", [(1, 512, 300), (37, 1000, 257), (700, 640, 1500)])
def test_captured_and_replayed_with_other_inputs(t, c, n):
    torch, L = _torch(), _learner()
    states = [_state(t, c, n, 1), _state(t, c, n, 2)]
    want = [[v.clone() for v in _step(L, *s)] for s in states]
    held = _state(t, c, n, 1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        _step(L, *held)
    side.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]     # two of them over the same buffers and the same pool
    outs, pool = [], torch.cuda.graph_pool_handle()
    for g in graphs:
        with torch.cuda.graph(g, pool=pool, stream=side):
            outs.append(_step(L, *held))
    for k in (1, 0, 1):
        for i in (0, 1):
            held[i].copy_(states[k][i])
        held[2].copy_(states[k][2])
        for i in (3, 4):
            held[i].codes.copy_(states[k][i].codes)
            held[i].scales.copy_(states[k][i].scales)
        for g, out in zip(graphs, outs):
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want[k]))
    L.sync()


def test_two_threads_on_streams_of_their_own():
    torch, L = _torch(), _learner()
    shapes = [(300, 512, 400), (40, 1000, 129)]
    states = [_state(*shape, 7 + i) for i, shape in enumerate(shapes)]
    want = [[v.clone() for v in _step(L, *s)] for s in states]
    torch.cuda.synchronize()
    failed = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got = _step(L, *states[i])
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                        failed.append(i)
                L.sync()
        except Exception as exc:      # noqa: BLE001
            failed.append(exc)

    threads = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not failed


@pytest.mark.parametrize("blocks", range(1, 10))
def test_few_rows_by_clusters_of_every_size(blocks):
    # 8 rows of 1000 columns to a block
    torch, L = _torch(), _learner()
    t = 8 * blocks - 3
    rng = np.random.default_rng(blocks)
    dy, s, w = (rng.standard_normal(shape).astype(np.float32) for shape in ((t, 1000), (t, 1000), 1000))
    ds, dw = L.rms_norm_backward(*(torch.from_numpy(v).cuda() for v in (dy, s, w)))
    want, want_w, size, size_w = ref.norm_backward(dy, s, w, 1e-6)
    _close(_np(ds), want, 100 * U * size)
    _close(_np(dw), want_w, (t + 65) * U * size_w)


def test_pull_norm_and_product_around_a_busy_stream():
    # the server on the legacy stream; a long line of work on the learner's before a pull that is used at once
    torch, L = _torch(), _learner()
    from paper_1509_04210_b200 import binding as rb
    theta = torch.randn(300 * 512, device="cuda") * 0.05
    ps = rb.ParameterServer(theta.numel(), 1, 1, 0.1)
    ps.set_weights(theta)
    ps.sync()
    x, w = torch.randn(20, 512, device="cuda").bfloat16(), torch.ones(512, device="cuda")
    want = L.fp8_matmul(L.rms_norm(x, w, fp8=True), L.fp8_quantize(theta.view(300, 512), square=True))
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for _ in range(3):
            torch.cuda._sleep(100_000_000)
            q, _ = L.pull_fp8(ps, 0, 300, 512)
            assert torch.equal(L.fp8_matmul(L.rms_norm(x, w, fp8=True), q), want)
            del q
    ps.close()
