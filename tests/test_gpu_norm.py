"""The norm with the residual's addition, forward and backward, on the GPU against its definition in 64 bits.

Tolerances, u = 2^-24 (half a step of float32).  A sum of c squares: at most 16 roundings within a thread's piece, one for each
further piece (c / 4096 of them at most) and 10 where threads meet, relative to a sum of positive terms; the inverse root takes half
of that, and adds its own, the mean's and eps's: (13 + c / 8192 + 3) u.  y adds two products: within (18 + c / 8192) u, taken as
(32 + c / 8192) u of itself.  The mean of w dy s is off by (17 + c / 4096 + 10) u of the mean of magnitudes; ds by
at most twice that and five roundings of the sum of magnitudes of its parts: (96 + c / 1024) u.  dw: as many roundings as
tokens and a few where parts meet, and the inverse root's: (t + 64 + c / 8192) u of the sum of magnitudes.  Outputs of bf16 add half a step, 2^-8."""
import numpy as np
import pytest

import block_reference as ref
from test_gpu_learner import _close, _dev, _learner, _normal, _np, _torch

pytestmark = pytest.mark.gpu
U, EPS = 2.0 ** -24, 1e-6

SHAPES = [(1, 1), (1, 15), (3, 16), (2, 17), (5, 128), (1, 129), (37, 1000), (7, 512), (4, 513), (130, 260), (3, 4096), (2, 4111), (300, 64), (9, 8192), (3, 8193), (2, 9216), (2, 16400), (1, 40000),
          (1000, 33)]


def _inputs(t, c, dtype, weight, pad, shift, residual=True):
    x, hx = _dev(_normal(t, c, 0.7, 1), dtype, pad, shift)
    r, hr = _dev(_normal(t, c, 2.0, 2), dtype, pad, shift) if residual else (None, 0.0)
    w, hw = _dev(1.0 + _normal(1, c, 0.2, 3), weight, 0, shift)
    s = (hx + hr).astype(np.float32)
    if dtype == "bf16":
        s = _torch().from_numpy(s).bfloat16().float().numpy()
    return x, r, w[0], s, hw[0]


def _half(dtype, v):
    return 2.0 ** -8 * np.abs(v) if dtype == "bf16" else 0.0


def _fp8_near(q, y, tol):
    """Values of FP8 within half a step of y, give or take tol: 1/16 of the value, 2^-10 of the scale; a scale may be the next
    larger or smaller one where the block's largest value is within tol of the border."""
    v = _np(_learner().fp8_dequantize(q, _torch().float32))
    top = np.zeros_like(y)
    for b in range(0, y.shape[1], 128):
        top[:, b:b + 128] = np.abs(y[:, b:b + 128]).max(axis=1, keepdims=True)
    _close(v, y, np.maximum(np.abs(y) * (1 + tol) / 16, top / 224 * (1 + 2 * tol) * 2.0 ** -10) + tol * np.abs(y) + 2.0 ** -149)


@pytest.mark.parametrize("t,c", SHAPES)
@pytest.mark.parametrize("dtype,weight,pad,shift", [("f32", "f32", 0, 0), ("bf16", "f32", 0, 0), ("bf16", "bf16", 8, 0), ("f32", "bf16", 3, 1), ("bf16", "f32", 3, 5)])
def test_forward(t, c, dtype, weight, pad, shift):
    torch, L = _torch(), _learner()
    x, r, w, s, hw = _inputs(t, c, dtype, weight, pad, shift)
    tol = (32 + c / 8192) * U
    y, total = L.rms_norm(x, w, r, eps=EPS)
    np.testing.assert_array_equal(_np(total), s.astype(np.float64))       # one rounding
    want = ref.norm(s, hw, EPS)
    _close(_np(y), want, tol * np.abs(want) * (1 + 2.0 ** -8) + _half(dtype, want))
    y8, total8, kept = L.rms_norm(x, w, r, eps=EPS, fp8=True, keep=True)
    assert torch.equal(total8, total)
    _fp8_near(y8, want, tol)
    if dtype == "f32":                  # y itself was written: the other forms are those of it
        q, a = L.fp8_quantize(y), L.act8_save(y)
        assert torch.equal(y8.codes, q.codes) and torch.equal(L.fp8_dequantize(y8), L.fp8_dequantize(q))
        assert torch.equal(kept.codes, a.codes) and torch.equal(L.act8_values(kept), L.act8_values(a))
    else:
        v = _np(L.act8_values(kept, torch.float32))
        for b in range(0, c, 32):
            top = np.abs(want[:, b:b + 32]).max(axis=1, keepdims=True)
            _close(v[:, b:b + 32], want[:, b:b + 32], top / 127 * (1 + tol) + tol * top + 2.0 ** -149)
    # no residual: of the sum itself
    plain, kept2 = L.rms_norm(total, w, eps=EPS, keep=True)
    assert torch.equal(plain, y) and torch.equal(kept2.codes, kept.codes)


@pytest.mark.parametrize("c", [100, 1000, 4096, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_in_place_and_around_the_outputs(c, dtype):
    torch, L = _torch(), _learner()
    x, r, w, s, hw = _inputs(5, c, dtype, "f32", 3, 1)
    y, total = L.rms_norm(x, w, r)
    for which in (x, r):
        other = r if which is x else x
        buf = torch.full((7, c + 9), 7.0, dtype=x.dtype, device="cuda")
        place = buf[1:6, 4:c + 4]
        place.copy_(which)
        out = torch.full((7, c + 9), 7.0, dtype=x.dtype, device="cuda")
        y2, total2 = L.rms_norm(place, w, other, out=out[1:6, 3:c + 3], out_sum=place) if which is x else L.rms_norm(other, w, place, out=out[1:6, 3:c + 3], out_sum=place)
        assert torch.equal(y2, y) and torch.equal(place, total) and total2.data_ptr() == place.data_ptr()
        for b, at in ((buf, 4), (out, 3)):
            assert (b[0] == 7).all() and (b[6] == 7).all() and (b[:, :at] == 7).all() and (b[:, at + c:] == 7).all()
    alone = total.clone()
    L.rms_norm(alone, w, out=alone)
    assert torch.equal(alone, y)


def test_rows_of_zeros_of_large_and_of_non_finite_values():
    torch, L = _torch(), _learner()
    x = _normal(8, 300, 1.0)
    x[1] = 0.0
    x[2] *= 1e17
    x[3] *= 1e-17
    x[4, 7] = np.nan
    x[5, 7] = np.inf
    w = np.ones(300, dtype=np.float32)
    d = torch.from_numpy(x).cuda()
    y = _np(L.rms_norm(d, torch.ones(300, device="cuda"), eps=EPS))
    rows = [0, 1, 2, 3, 6, 7]
    want = ref.norm(x[rows], w, EPS)
    _close(y[rows], want, 40 * U * np.abs(want))
    assert np.isnan(y[4]).all() and np.isnan(y[5, 7]) and (np.delete(y[5], 7) == 0).all()
    q = L.rms_norm(d, torch.ones(300, device="cuda"), fp8=True)
    v = _np(L.fp8_dequantize(q))
    assert np.isnan(v[4]).all() and np.isnan(v[5, :128]).all() and (v[5, 128:] == 0).all() and (v[1] == 0).all()


@pytest.mark.parametrize("t,c", SHAPES + [(600, 1000), (2500, 130)])
@pytest.mark.parametrize("dtype,weight,pad,shift", [("f32", "f32", 0, 0), ("bf16", "f32", 0, 0), ("bf16", "bf16", 8, 0), ("f32", "bf16", 3, 1), ("bf16", "f32", 3, 5)])
@pytest.mark.parametrize("through", [True, False])
def test_backward(t, c, dtype, weight, pad, shift, through):
    torch, L = _torch(), _learner()
    s, _, w, hs, hw = _inputs(t, c, dtype, weight, pad, shift, residual=False)
    dy, hdy = _dev(_normal(t, c, 1e-3, 5), dtype, pad, shift)
    more, hmore = _dev(_normal(t, c, 1e-3, 6), dtype, 0, shift) if through else (None, None)
    ds, dw = L.rms_norm_backward(dy, s, w, eps=EPS, dsum=more)
    want, want_w, size, size_w = ref.norm_backward(hdy, hs, hw, EPS, hmore)
    _close(_np(ds), want, (96 + c / 1024) * U * size + _half(dtype, want))
    tol_w = (t + 64 + c / 8192) * U * size_w
    assert dw.dtype == torch.float32
    _close(_np(dw), want_w, tol_w)
    # the weight's gradient where it is pushed from, the input's over what it is computed from
    vector = torch.full((c + 20,), 7.0, dtype=torch.bfloat16, device="cuda")
    over = dy.clone() if not through else more
    ds2, dw2 = L.rms_norm_backward(over if not through else dy, s, w, eps=EPS, dsum=more, out=over, out_weight=vector[7:7 + c])
    assert torch.equal(ds2, ds) and ds2.data_ptr() == over.data_ptr() and dw2.data_ptr() == vector[7:].data_ptr()
    _close(_np(vector[7:7 + c]), want_w, tol_w * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want_w))
    assert (vector[:7] == 7).all() and (vector[7 + c:] == 7).all()
    again = dy.clone()
    assert all(torch.equal(a, b) for a, b in zip(L.rms_norm_backward(again, s, w, eps=EPS), L.rms_norm_backward(again, s, w, eps=EPS, out=again)))


#: enough rows to go through rings, at widths that fill a warp, a part of one, several, and more than a block's
LONG = [(7200, 504), (8000, 40), (3000, 1000), (2000, 4096), (1400, 4112), (1000, 8200), (700, 9216)]


@pytest.mark.parametrize("t,c", LONG)
@pytest.mark.parametrize("pad", [0, 8])
def test_many_rows(t, c, pad):
    torch, L = _torch(), _learner()
    x, r, w, s, hw = _inputs(t, c, "bf16", "f32", pad, 0)
    tol = (32 + c / 8192) * U
    want = ref.norm(s, hw, EPS)
    for residual in (True, False):
        got = L.rms_norm(x, w, r, eps=EPS) if residual else (L.rms_norm(torch.from_numpy(s).cuda().bfloat16(), w, eps=EPS), None)
        _close(_np(got[0]), want, tol * np.abs(want) * (1 + 2.0 ** -8) + _half("bf16", want))
        assert not residual or np.array_equal(_np(got[1]), s.astype(np.float64))
    y8, total, kept = L.rms_norm(x, w, r, eps=EPS, fp8=True, keep=True)
    _fp8_near(y8, want, tol)
    # (few rows by themselves need not give the same codes: their squares are added in another order, within the same bound, and a
    # value of y that is nearly half way between two codes may fall to either)
    v = _np(L.act8_values(kept, torch.float32))
    top = np.repeat(np.abs(np.pad(want, ((0, 0), (0, -c % 32)))).reshape(t, -1, 32).max(axis=2), 32, axis=1)[:, :c]
    _close(v, want, top / 127 * (1 + tol) + tol * top + 2.0 ** -149)
    dy, hdy = _dev(_normal(t, c, 1e-3, 5), "bf16", pad)
    more, hmore = _dev(_normal(t, c, 1e-3, 6), "bf16", 0)
    sums, hs = _dev(s, "bf16", pad)
    for m, hm in ((more, hmore), (None, None)):
        ds, dw = L.rms_norm_backward(dy, sums, w, eps=EPS, dsum=m)
        want_d, want_w, size, size_w = ref.norm_backward(hdy, hs, hw, EPS, hm)
        _close(_np(ds), want_d, (96 + c / 1024) * U * size + _half("bf16", want_d))
        _close(_np(dw), want_w, (t + 64 + c / 8192) * U * size_w)
        again = L.rms_norm_backward(dy, sums, w, eps=EPS, dsum=m, out=m)
        assert torch.equal(again[0], ds) and torch.equal(again[1], dw)
    L.sync()


def test_backward_against_differences():
    """The change of sum(g * y) along a direction, from the forward kernel, against the backward kernel's.  With steps of h = 2^-6 of values
    near 1 the central difference is off by h^2 / 6 of third derivatives (a few units each for x, none for w), and by rounding, (32 U) / h of
    the sum of magnitudes."""
    torch, L = _torch(), _learner()
    t, c, h = 6, 200, 2.0 ** -6
    s, w, g = (torch.from_numpy(_normal(a, c, d, k)).cuda() for a, d, k in ((t, 1.0, 1), (1, 0.2, 2), (t, 1.0, 3)))
    w = w[0] + 1
    us, uw = torch.from_numpy(_normal(t, c, 1.0, 4)).cuda(), torch.from_numpy(_normal(1, c, 1.0, 5)).cuda()[0]
    ds, dw = L.rms_norm_backward(g, s, w, eps=EPS)
    f = lambda a, b: (L.rms_norm(a, b, eps=EPS).double() * g.double()).sum().item()  # noqa: E731
    size = (g.double() * L.rms_norm(s, w, eps=EPS).double()).abs().sum().item()
    by_s = (f(s + h * us, w) - f(s - h * us, w)) / (2 * h)
    by_w = (f(s, w + h * uw) - f(s, w - h * uw)) / (2 * h)
    assert abs(by_s - (ds.double() * us.double()).sum().item()) < size * (32 * U / h + h * h * 4)
    assert abs(by_w - (dw.double() * uw.double()).sum().item()) < size * 64 * U / h


def test_empty_sizes_and_refusals():
    torch, L = _torch(), _learner()
    w = torch.ones(64, device="cuda")
    e = torch.empty(0, 64, device="cuda")
    assert L.rms_norm(e, w).shape == (0, 64) and [v.shape for v in L.rms_norm(e, w, e)] == [(0, 64)] * 2
    ds, dw = L.rms_norm_backward(e, e, w)
    assert ds.shape == (0, 64) and (dw == 0).all()
    n = torch.empty(3, 0, device="cuda")
    assert L.rms_norm(n, w[:0]).shape == (3, 0) and L.rms_norm_backward(n, n, w[:0])[1].shape == (0,)
    x = torch.ones(4, 64, device="cuda")
    from paper_1509_04210_b200 import binding as rb
    for call in (lambda: L.rms_norm(x, w[:63]), lambda: L.rms_norm(x, w.view(1, 64)), lambda: L.rms_norm(x, w.half()), lambda: L.rms_norm(x, w, x[:3]),
                 lambda: L.rms_norm(x, w, x.bfloat16()), lambda: L.rms_norm(x, w, out_sum=x), lambda: L.rms_norm(x, w, out=x.bfloat16()), lambda: L.rms_norm(x, w, fp8=True, out=x),
                 lambda: L.rms_norm(x, w, out=L.fp8_quantize(x)), lambda: L.rms_norm(x, w, saved=L.fp8_quantize(x)), lambda: L.rms_norm(x, w.cpu()), lambda: L.rms_norm(x.t(), w[:4]),
                 lambda: L.rms_norm(x, torch.ones(128, device="cuda")[::2]), lambda: L.rms_norm(x.clone().requires_grad_(), w), lambda: L.rms_norm(x, w.clone().requires_grad_()),
                 lambda: L.rms_norm_backward(x[:3], x, w), lambda: L.rms_norm_backward(x.bfloat16(), x, w), lambda: L.rms_norm_backward(x, x, w, dsum=x[:, :63]),
                 lambda: L.rms_norm_backward(x, x, w, out_weight=w[:63]), lambda: L.rms_norm_backward(x, x, w, dtype=torch.float16), lambda: L.rms_norm_backward(x, x, w, out=x.bfloat16())):
        with pytest.raises(ValueError):
            call()
    for eps in (-1e-6, float("nan"), float("inf")):
        with pytest.raises(rb.RudraError, match="eps"):
            L.rms_norm(x, w, eps=eps)
        with pytest.raises(rb.RudraError, match="eps"):
            L.rms_norm_backward(x, x, w, eps=eps)
