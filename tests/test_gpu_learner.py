"""The learner-side operators on the GPU, through the public interface, against 64-bit definitions.

Codes and scales are compared exactly (scales are powers of two, so nothing in them depends on the
precision of the arithmetic).  Tolerances of the computed numbers follow from the operators:

* a sum of K exact products in 32 bits is within K * 2^-23 of the sum of their magnitudes (K additions,
  each off by at most one unit in the last place, truncating units included);
* x * sigmoid(z) is within (8 + 4 |z|) * 2^-23 of its magnitude: the exponential's argument is rounded
  (|z| * 2^-24 of it, twice), exponential and reciprocal are within 2 units each, two products follow;
* an output in bf16 adds half a unit in its last place, 2^-8 of the value at most.
"""
import numpy as np
import pytest

import learner_reference as ref

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -23


def _torch():
    import torch
    return torch


def _learner():
    from paper_1509_04210_b200 import learner
    return learner


def _dev(x, dtype="f32", pad=0, shift=0):
    """A matrix on the GPU whose rows are cols + pad apart and start `shift` elements into the buffer,
    with NaN around it; and the float32 values it holds."""
    torch = _torch()
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rows, cols = x.shape
    buf = torch.full((shift + rows * (cols + pad),), float("nan"), dtype=t, device="cuda")
    view = buf[shift:].view(rows, cols + pad)[:, :cols]
    view.copy_(torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda())
    return view, view.float().cpu().numpy()


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _rng(*key):
    return np.random.default_rng([20150914] + [int(k) for k in key])


def _normal(rows, cols, std=1.0, key=0):
    return (_rng(rows, cols, key).standard_normal((rows, cols)) * std).astype(np.float32)


def _close(got, want, tol):
    same = np.isnan(got) & np.isnan(want)
    off = np.where(same, 0.0, np.abs(got - want))
    assert not np.isnan(off).any(), "NaN on one side only"
    worst = np.unravel_index(np.argmax(off - tol), off.shape) if off.size else None
    assert off.size == 0 or (off <= tol).all(), (worst, got[worst], want[worst], off[worst], np.broadcast_to(tol, off.shape)[worst])


# ------------------------------------------------------------------------------------------- MX4

SHAPES = [(1, 1), (1, 31), (3, 32), (1, 33), (2, 127), (5, 128), (7, 129), (130, 260), (33, 1000), (129, 64), (257, 95), (64, 4096)]


def _check_mx4(q, x):
    codes, scales = ref.mx4_bytes(x)
    rows, cols = x.shape
    assert (q.rows, q.cols) == (rows, cols)
    np.testing.assert_array_equal(q.codes.cpu().numpy().reshape(codes.shape), codes)
    nb = -(-cols // 32)
    kt = -(-nb // 4)
    r, b = np.meshgrid(np.arange(rows), np.arange(4 * kt), indexing="ij")
    at = ref.mx4_scale_at(r, b, kt)          # padding blocks of a row included, padding rows not
    np.testing.assert_array_equal(q.scales.cpu().numpy()[at], scales[at])


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype,pad,shift", [("f32", 0, 0), ("bf16", 0, 0), ("f32", 3, 1), ("bf16", 8, 5)])
@pytest.mark.parametrize("transpose", [False, True])
def test_quantize_is_exact(rows, cols, dtype, pad, shift, transpose):
    L = _learner()
    x, held = _dev(_normal(rows, cols, 0.01), dtype, pad, shift)
    q = L.mx4_quantize(x, transpose)
    held = held.T if transpose else held
    _check_mx4(q, held)
    want = ref.mx4_values(held)
    for out in (_torch().float32, _torch().bfloat16):
        np.testing.assert_array_equal(_np(L.mx4_dequantize(q, out)), want)


def test_quantize_ties_saturation_and_signs():
    L = _learner()
    grid = np.concatenate([ref.GRID, (ref.GRID[1:] + ref.GRID[:-1]) / 2, [6.5, 7.0, 7.9]])
    fine = np.concatenate([grid, np.nextafter(grid.astype(np.float32), np.float32(9)), np.nextafter(grid.astype(np.float32), np.float32(-9))])
    fine = fine[fine < 8]
    row = np.zeros((len(fine) * 2, 32), dtype=np.float32)
    row[:, 0] = 4.0                       # fixes the scale at 1
    row[:, 1] = np.concatenate([fine, -fine])
    row[:, 2] = -0.0
    for scale in (1.0, 2.0 ** -120, 2.0 ** 120):
        x = (row * np.float32(scale)).astype(np.float32)
        q = L.mx4_quantize(_dev(x)[0])
        _check_mx4(q, x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("transpose", [False, True])
def test_extreme_and_non_finite_blocks(dtype, transpose):
    L = _learner()
    x = _normal(40, 32 * 11, 1.0)
    big, tiny = np.float32(3.3895314e38), np.float32(2.0 ** -133)
    x[1, 0:32] = 0.0
    x[2, 40] = np.inf
    x[3, 70] = -np.inf
    x[4, 100] = np.nan
    x[5, 130:140] = big
    x[6, 160:192] = tiny
    x[7, 192:224] = tiny
    x[7, 193] = np.float32(2.0 ** -126)
    x[8, 224:256] = np.float32(2.0 ** -125)
    x[9, 256:288] = -big
    x[10] = 0.0
    x[11] = np.nan
    v, held = _dev(x, dtype)
    held = held.T if transpose else held
    q = L.mx4_quantize(v, transpose)
    _check_mx4(q, held)
    np.testing.assert_array_equal(_np(L.mx4_dequantize(q, _torch().float32)), ref.mx4_values(held))
    if not transpose:
        saved = L.act8_save(v)
        codes, s = ref.act8(held)
        np.testing.assert_array_equal(saved.scales.cpu().numpy()[:, :s.shape[1]], s)
        np.testing.assert_array_equal(saved.codes.cpu().numpy(), codes)
        np.testing.assert_array_equal(_np(L.act8_values(saved, _torch().float32)), ref.act8_values(held))


def _product(a, b):
    """(a b^T, the same of magnitudes) in 64 bits."""
    if a.shape[0] * b.shape[0] * a.shape[1] < 1e9:
        return a @ b.T, np.abs(a) @ np.abs(b).T
    torch = _torch()                                     # the same, sooner
    a, b = torch.from_numpy(a).cuda(), torch.from_numpy(b).cuda()
    return (a @ b.t()).cpu().numpy(), (a.abs() @ b.abs().t()).cpu().numpy()


def _check_product(got, a, b, bf16):
    want, size = _product(a, b)
    _close(_np(got), want, a.shape[1] * EPS * size + (2.0 ** -8 * np.abs(want) if bf16 else 0.0))


# rows of x, outputs, inner length: single rows to several tiles, every kind of ragged edge
PRODUCTS = [(1, 1, 1), (1, 8, 32), (1, 129, 33), (2, 64, 64), (3, 1000, 65), (8, 200, 257), (16, 128, 512), (17, 130, 500), (33, 31, 4096),
            (64, 384, 640), (65, 257, 96), (100, 1000, 512), (128, 128, 256), (129, 127, 1000), (200, 513, 288), (256, 256, 1024),
            (300, 260, 2080), (513, 640, 384), (1, 4096, 9216), (5, 1000, 4096),
            # enough tiles for pairs of blocks: ragged in every direction, one stage and many
            (2305, 2049, 33), (2310, 2050, 1000), (2560, 2304, 256), (4100, 1300, 130), (1281, 4000, 2200)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_product_against_the_definition(m, n, k, dtype):
    L, torch = _learner(), _torch()
    x, xh = _dev(_normal(m, k, 1.0, 1), dtype, pad=3 if m % 2 else 0)
    w, wh = _dev(_normal(n, k, 0.01, 2))
    q = L.mx4_quantize(w)
    a, b = ref.mx4_values(xh), ref.mx4_values(wh)
    out = torch.float32 if dtype == "f32" else torch.bfloat16
    got = L.mx4_matmul(x, q, out)
    _check_product(got, a, b, dtype == "bf16")
    # the same from codes, into a view with canaries around it
    hold = torch.full((m + 2, n + 5), 7.0, dtype=out, device="cuda")
    L.mx4_matmul(L.mx4_quantize(x), q, out=hold[1:m + 1, 2:n + 2])
    assert torch.equal(hold[1:m + 1, 2:n + 2], got)
    hold[1:m + 1, 2:n + 2] = 7.0
    assert bool((hold == 7.0).all())


def test_product_does_not_depend_on_the_run_or_the_batch():
    L, torch = _learner(), _torch()
    x, _ = _dev(_normal(300, 9216, 1.0, 3), "bf16")
    q = L.mx4_quantize(_dev(_normal(1000, 9216, 0.01, 4))[0])
    first = L.mx4_matmul(x, q, torch.float32)
    for _ in range(3):
        assert torch.equal(L.mx4_matmul(x, q, torch.float32), first)


def test_product_with_blocks_of_nan_and_zero():
    L, torch = _learner(), _torch()
    x = _normal(40, 320, 1.0, 5)
    w = _normal(200, 320, 1.0, 6)
    x[3, 40] = np.nan
    x[5] = 0.0
    w[7, 300] = np.inf
    w[11] = 0.0
    xd, wd = _dev(x)[0], _dev(w)[0]
    got = _np(L.mx4_matmul(xd, L.mx4_quantize(wd), torch.float32))
    a, b = ref.mx4_values(x), ref.mx4_values(w)
    with np.errstate(invalid="ignore"):
        want, size = _product(a, b)
    _close(got, want, 320 * EPS * np.where(np.isnan(size), 0.0, size))
    assert np.isnan(got[3]).all() and np.isnan(got[:, 7]).all() and (np.delete(got[5], 7) == 0).all()


def test_product_of_extreme_scales():
    # scales multiply: 2^100 * 2^-100 must not overflow or vanish on the way
    L, torch = _learner(), _torch()
    x = _normal(20, 256, 1.0, 7) * np.float32(2.0 ** 100)
    w = _normal(64, 256, 1.0, 8) * np.float32(2.0 ** -100)
    got = L.mx4_matmul(_dev(x)[0], L.mx4_quantize(_dev(w)[0]), torch.float32)
    _check_product(got, ref.mx4_values(x), ref.mx4_values(w), False)


@pytest.mark.parametrize("m,n,k", [(0, 5, 32), (5, 0, 32), (4, 6, 0), (0, 0, 0), (200, 130, 0)])
def test_product_of_nothing(m, n, k):
    L, torch = _learner(), _torch()
    x = torch.zeros((m, k), device="cuda")
    q = L.mx4_quantize(torch.zeros((n, k), device="cuda"))
    got = L.mx4_matmul(x, q, out=torch.full((m, n), 3.0, device="cuda"))
    assert got.shape == (m, n) and bool((got == 0).all())


# --------------------------------------------------------------------------------- checkpoints

ACTS = ["relu", "silu", "gelu", "swiglu"]


def _act_tol(act, x, size, bf16):
    with np.errstate(over="ignore", invalid="ignore"):
        z = np.minimum(np.abs(ref.sigmoid_argument(act, x)), 200.0)
    return (8 + 4 * z) * EPS * size + (2.0 ** -8 * size if bf16 else 0.0) + 2.0 ** -126


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (2, 1000), (37, 257), (5, 4096)])
@pytest.mark.parametrize("dtype,pad,shift", [("f32", 0, 0), ("bf16", 0, 0), ("f32", 5, 3), ("bf16", 8, 1)])
def test_activation_and_checkpoint(act, rows, cols, dtype, pad, shift):
    L, torch = _learner(), _torch()
    two = act == "swiglu"
    x, xh = _dev(_normal(rows, cols, 2.0, 1), dtype, pad, shift)
    u, uh = _dev(_normal(rows, cols, 2.0, 2), dtype, pad, shift)
    dy, dyh = _dev(_normal(rows, cols, 1e-3, 3), dtype, 1, 2)
    res = L.act8_forward(act, x, *([u] if two else []))
    y, saved = res[0], res[1]
    xd, ud, g = xh.astype(np.float64), uh.astype(np.float64), dyh.astype(np.float64)
    bf = dtype == "bf16"
    want = ref.f(act, xd) * (ud if two else 1.0)
    size = np.abs(xd) * ref.sigmoid(ref.sigmoid_argument(act, xd)) * (np.abs(ud) if two else 1.0) if act != "relu" else np.abs(want)
    _close(_np(y), want, _act_tol(act, xd, size, bf))
    for s, h in ((saved, xh), (res[2], uh)) if two else ((saved, xh),):
        codes, scale = ref.act8(h)
        got = s.codes.cpu().numpy()
        np.testing.assert_array_equal(got[:, :cols], codes)
        assert not got[:, cols:].any()
        np.testing.assert_array_equal(s.scales.cpu().numpy()[:, :scale.shape[1]], scale)
        np.testing.assert_array_equal(_np(L.act8_values(s, torch.bfloat16)), ref.act8_values(h))
    xq, uq = ref.act8_values(xh), ref.act8_values(uh)
    d = ref.slope(act, xq)
    # the slope is a sum of terms of size 1 and |x s (1 - s) u'|; errors are relative to those
    s = ref.sigmoid(ref.sigmoid_argument(act, xq))
    du = 2 * ref.GELU_A * (1 + 3 * ref.GELU_B * xq ** 2) if act == "gelu" else 1.0
    terms = 1.0 + np.abs(xq) * s * (1 - s) * du
    back = L.act8_backward(act, dy, saved, *([res[2]] if two else []))
    dx = back[0] if two else back
    k = np.abs(g) * (np.abs(uq) if two else 1.0)
    rounding = 2.0 ** -8 * np.abs(g * d * (uq if two else 1.0)) if bf else 0.0
    _close(_np(dx), g * d * (uq if two else 1.0), _act_tol(act, xq, k * terms, False) * 2 + rounding)
    if two:
        wu = g * ref.f(act, xq)
        _close(_np(back[1]), wu, _act_tol(act, xq, np.abs(wu), bf))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_slope_against_differences(act):
    # the gradient the backward pass applies is the derivative of the forward function at the saved value
    L, torch = _learner(), _torch()
    x, xh = _dev(_normal(16, 512, 3.0, 4))
    _, saved = L.act8_forward(act, x)
    dx = _np(L.act8_backward(act, torch.ones_like(x), saved))
    xq, h = ref.act8_values(xh), 1e-5
    want = (ref.f(act, xq + h) - ref.f(act, xq - h)) / (2 * h)       # off by h^2 f''' / 6 < 1e-10 and 2^-52 |f| / h < 1e-9
    _close(dx, want, 1e-8 + 2 * _act_tol(act, xq, 1.0 + np.abs(xq), False))


def test_activations_far_out():
    L, torch = _learner(), _torch()
    x = np.zeros((4, 64), dtype=np.float32)
    x[0, :8] = [1e30, -1e30, 100.0, -100.0, 88.0, -88.0, 20.0, -20.0]
    x[1, :4] = [3e38, -3e38, 0.0, -0.0]
    x[2, 0], x[3, 40] = np.nan, np.inf
    xd, _ = _dev(x)
    for act in ("relu", "silu", "gelu"):
        y, saved = L.act8_forward(act, xd)
        got = _np(y)
        with np.errstate(over="ignore", invalid="ignore"):
            want = ref.f(act, x.astype(np.float64))
        finite = np.isfinite(x)
        np.testing.assert_allclose(got[finite], want[finite], rtol=1e-4, atol=1e-30)
        dx = _np(L.act8_backward(act, torch.ones_like(xd), saved))
        assert np.isnan(dx[2, :32]).all() and np.isnan(dx[3, 32:]).all()      # their blocks
        assert np.isfinite(dx[0]).all() and np.isfinite(dx[1]).all() and np.isfinite(dx[2, 32:]).all()
        assert dx[0, 0] == 1.0 and dx[0, 1] == 0.0 and dx[1, 0] == 1.0 and dx[1, 1] == 0.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(9, 300, 0, 0), (700, 1001, 0, 0), (300, 515, 3, 1)])
def test_gradient_may_overwrite_dy(dtype, rows, cols, pad, shift):
    L, torch = _learner(), _torch()
    x, _ = _dev(_normal(rows, cols, 1.0, 5), dtype)
    dy, _ = _dev(_normal(rows, cols, 1.0, 6), dtype, pad, shift)
    _, saved = L.act8_forward("gelu", x)
    want = L.act8_backward("gelu", dy, saved)
    L.act8_backward("gelu", dy, saved, out=dy)
    assert torch.equal(dy, want)


@pytest.mark.parametrize("shape", [(0, 32), (5, 0)])
def test_empty_activations(shape):
    L, torch = _learner(), _torch()
    x = torch.zeros(shape, device="cuda")
    y, saved = L.act8_forward("silu", x)
    assert y.shape == shape and L.act8_backward("silu", x, saved).shape == shape and L.act8_values(saved).shape == shape


# -------------------------------------------------------------------------------- weight gradient

# tokens, outputs, inputs
GRADS = [(1, 1, 1), (1, 40, 33), (2, 8, 31), (7, 130, 64), (31, 64, 100), (64, 128, 256), (65, 127, 257), (100, 1000, 96), (128, 129, 512),
         (300, 260, 1000), (509, 72, 640), (1000, 384, 130), (2048, 136, 264), (4100, 33, 40),
         # enough tiles for pairs of blocks
         (1, 2304, 2305), (65, 2050, 2400), (321, 1290, 4000), (600, 4097, 1281)]


@pytest.mark.parametrize("t,n,k", GRADS)
@pytest.mark.parametrize("dtype,pad,shift,out", [("bf16", 0, 0, "f32"), ("f32", 0, 0, "f32"), ("bf16", 3, 1, "bf16"), ("f32", 1, 1, "bf16"),
                                                 ("bf16", 8, 8, "f32")])
def test_weight_gradient_against_the_definition(t, n, k, dtype, pad, shift, out):
    L, torch = _learner(), _torch()
    x, xh = _dev(_normal(t, k, 1.0, 1), "bf16")
    dy, dyh = _dev(_normal(t, n, 1e-3, 2), dtype, pad, shift)
    saved = L.act8_save(x)
    kind = torch.float32 if out == "f32" else torch.bfloat16
    got = L.act8_weight_grad(dy, saved, kind)
    g, xq = dyh.astype(np.float64), ref.act8_values(xh)
    want, size = _product(np.ascontiguousarray(g.T), np.ascontiguousarray(xq.T))
    _close(_np(got), want, _sum_tol(t, out) * size + (2.0 ** -8 * np.abs(want) if out == "bf16" else 0.0))
    # the same, written into a flat vector that is to be pushed, at an odd place, with canaries around it
    flat = torch.full((n * k + 20,), 7.0, dtype=kind, device="cuda")
    L.act8_weight_grad(dy, saved, out=flat[13:13 + n * k].view(n, k))
    assert torch.equal(flat[13:13 + n * k].view(n, k), got)
    assert bool((flat[:13] == 7.0).all()) and bool((flat[13 + n * k:] == 7.0).all())


def _sum_tol(t, out):
    """Error of a weight gradient's sum over t tokens, of the sum of magnitudes.  A step of 16 products is cut off below the
    last place of its largest term, 17 terms by half a unit each at most; an f32 result is gathered every 512
    tokens (32 steps, 9 units each at most), for f32 gradients every 128 (three times 8 steps), and the parts are
    added with half a unit each.  Never more than a unit for every token."""
    gathered = 288 + t // 128 + 1 if out == "f32" else 9 * (t // 16 + 1)
    return min(max(t, 8), gathered) * EPS


@pytest.mark.parametrize("t,kind", [(65_600, "bf16"), (1 << 20, "bf16"), (1 << 20, "f32"), (30_001, "f32")])
def test_bf16_weight_gradient_over_very_many_tokens(t, kind):
    # positive terms: a sum that is cut off at every step drifts.  Here it is gathered like an f32 result, so the two
    # differ by the one rounding to bf16.
    L, torch = _learner(), _torch()
    x = torch.rand((t, 40), device="cuda", generator=torch.Generator("cuda").manual_seed(1)) + 0.5
    dy = torch.rand((t, 12), device="cuda", generator=torch.Generator("cuda").manual_seed(2)) + 0.5
    dy = dy.to(torch.bfloat16 if kind == "bf16" else torch.float32)
    saved = L.act8_save(x)
    exact = L.act8_weight_grad(dy, saved)
    want = dy.double().T @ L.act8_values(saved, torch.float32).double()
    assert bool(((exact.double() - want).abs() <= _sum_tol(t, "f32") * want).all())
    assert torch.equal(L.act8_weight_grad(dy, saved, torch.bfloat16), exact.bfloat16())


def test_weight_gradient_is_the_derivative_of_the_layer():
    # L(W) = sum dy * (xhat W^T) is linear in W: its differences are exact, entry by entry
    L, torch = _learner(), _torch()
    x, xh = _dev(_normal(50, 40, 1.0, 8), "bf16")
    dy, dyh = _dev(_normal(50, 12, 1.0, 9), "bf16")
    got = _np(L.act8_weight_grad(dy, L.act8_save(x)))
    xq, g = ref.act8_values(xh), dyh.astype(np.float64)
    w = _rng(1).standard_normal((12, 40))
    for i, j in [(0, 0), (11, 39), (3, 17), (7, 31), (5, 32)]:
        d = np.zeros_like(w)
        d[i, j] = 0.5
        diff = np.sum(g * (xq @ (w + d).T)) - np.sum(g * (xq @ (w - d).T))
        assert abs(got[i, j] - diff) <= 50 * EPS * np.sum(np.abs(g[:, i] * xq[:, j])) + 1e-9


def test_weight_gradient_of_no_tokens_and_non_finite_blocks():
    L, torch = _learner(), _torch()
    none = L.act8_weight_grad(torch.zeros((0, 40), device="cuda", dtype=torch.bfloat16), L.act8_save(torch.zeros((0, 300), device="cuda")),
                              out=torch.full((40, 300), 5.0, device="cuda"))
    assert bool((none == 0).all())
    x = _normal(200, 320, 1.0, 10)
    x[150, 70] = np.inf
    xd, xh = _dev(x, "bf16")
    dy, dyh = _dev(_normal(200, 140, 1.0, 11), "bf16")
    got = _np(L.act8_weight_grad(dy, L.act8_save(xd)))
    assert np.isnan(got[:, 64:96]).all()
    keep = np.r_[0:64, 96:320]
    xq, g = ref.act8_values(xh), dyh.astype(np.float64)
    _close(got[:, keep], (g.T @ np.nan_to_num(xq))[:, keep], 200 * EPS * (np.abs(g).T @ np.abs(np.nan_to_num(xq)))[:, keep])


def test_weight_gradient_does_not_depend_on_the_run():
    L, torch = _learner(), _torch()
    x, _ = _dev(_normal(3000, 520, 1.0, 12), "bf16")
    dy, _ = _dev(_normal(3000, 250, 1.0, 13), "f32")
    saved = L.act8_save(x)
    first = L.act8_weight_grad(dy, saved)
    for _ in range(3):
        assert torch.equal(L.act8_weight_grad(dy, saved), first)


# ------------------------------------------------------------------------- streams, server, together

def test_operators_follow_the_current_stream():
    L, torch = _learner(), _torch()
    x, xh = _dev(_normal(64, 512, 1.0, 14), "bf16")
    w, wh = _dev(_normal(300, 512, 0.01, 15))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        busy = torch.randn(4096, 4096, device="cuda")
        for _ in range(20):
            busy = busy @ busy * 1e-3
        x2, w2 = x * 1.0, w * 1.0                        # inputs that exist only once the stream gets there
        y = L.mx4_matmul(x2, L.mx4_quantize(w2), torch.float32)
        dw = L.act8_weight_grad(x2, L.act8_save(x2))
    s.synchronize()
    _check_product(y, ref.mx4_values(xh), ref.mx4_values(wh), False)
    xq, g = ref.act8_values(xh), xh.astype(np.float64)
    _close(_np(dw), g.T @ xq, 64 * EPS * (np.abs(g).T @ np.abs(xq)))


def test_operators_can_be_captured_in_a_graph():
    L, torch = _learner(), _torch()
    x, _ = _dev(_normal(48, 1024, 1.0, 16), "bf16")
    q = L.mx4_quantize(_dev(_normal(256, 1024, 0.01, 17))[0])

    def step():
        y = L.mx4_matmul(x, q)
        z, saved = L.act8_forward("silu", y)
        return z, L.act8_weight_grad(L.act8_backward("silu", z, saved), L.act8_save(x))

    want = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    x.mul_(-1.0)
    graph.replay()
    fresh = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, fresh)) and not torch.equal(got[0], want[0])


@pytest.mark.parametrize("transpose", [False, True])
def test_pull_in_four_bits(transpose):
    L, torch = _learner(), _torch()
    from paper_1509_04210_b200 import binding as rb
    n, rows, cols, offset = 70001, 130, 260, 4097
    theta = torch.randn(n, device="cuda") * 0.01
    ps = rb.ParameterServer(n, 2, 1, 0.1)
    ps.set_weights(theta)
    grads = [torch.randn(n, device="cuda") * 0.01 for _ in range(2)]
    for g in grads:
        ps.push(g, 0)
    assert ps.step() == 1
    before = ps.counters()
    q, ts = L.pull_mx4(ps, offset, rows, cols, transpose)
    full = torch.empty(n, device="cuda")
    assert ts == ps.pull(full) == 1
    ps.sync()
    held = full[offset:offset + rows * cols].view(rows, cols).cpu().numpy()
    _check_mx4(q, held.T if transpose else held)
    assert ps.counters()["pulls"] == before["pulls"] + 2
    for bad in ((n - rows * cols + 1, rows, cols), (n + 1, 1, 1), (0, n, 2)):
        with pytest.raises(rb.RudraError) as e:
            ps.pull_mx4(*bad, False, q.codes, q.scales)
        assert e.value.code == rb.E_INVAL and "past the end" in str(e.value)
    with pytest.raises(rb.RudraError):
        ps.pull_mx4(0, 2, 2, False, None, q.scales)
    ps.close()


def test_refusals_on_the_gpu():
    L, torch = _learner(), _torch()
    from paper_1509_04210_b200 import binding as rb
    x = torch.zeros((4, 64), device="cuda")
    q = L.mx4_quantize(x)
    with pytest.raises(ValueError):
        L.mx4_quantize(x.double())
    with pytest.raises(ValueError):
        L.mx4_quantize(x.t())                                   # columns are not rows
    with pytest.raises(ValueError):
        L.mx4_quantize(x.cpu())
    with pytest.raises(ValueError):
        L.mx4_matmul(torch.zeros((4, 65), device="cuda"), q)
    with pytest.raises(ValueError):
        L.mx4_matmul(x, L.MX4(q.codes[:2], q.scales, 4, 64))    # fewer codes than the matrix has
    with pytest.raises(ValueError):
        L.mx4_matmul(x, q, out=torch.zeros((4, 5), device="cuda"))
    with pytest.raises(ValueError):
        L.act8_forward("tanh", x)
    with pytest.raises(ValueError):
        L.act8_forward("swiglu", x)
    with pytest.raises(ValueError):
        L.act8_forward("silu", x, x)
    with pytest.raises(ValueError):
        L.act8_weight_grad(torch.zeros((5, 64), device="cuda"), L.act8_save(x))
    assert L.sync() is None
    off = torch.zeros(4096, dtype=torch.uint8, device="cuda")[1:]
    with pytest.raises(rb.RudraError) as e:
        L.mx4_quantize(x, out=L.MX4(off, q.scales, 4, 64))      # codes not on a 32-byte boundary
    assert e.value.code == rb.E_INVAL and "32-byte" in str(e.value)


def test_matrices_of_more_than_2_to_the_32_values():
    # every offset on the way is 64 bits wide: rows from both ends and from around the boundaries have to come out
    # as they do by themselves
    L, torch = _learner(), _torch()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    rows, cols = 67000, 65536                                       # 4.39e9 values
    pick = torch.tensor([0, 1, 32767, 32768, 65535, 65536, rows - 2, rows - 1], device="cuda")
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    for r in range(0, rows, 8000):
        x[r:r + 8000].normal_()
    few = x[pick].contiguous()
    q = L.mx4_quantize(x)
    assert torch.equal(q.codes[pick], L.mx4_quantize(few).codes)
    back = L.mx4_dequantize(q)
    assert torch.equal(back[pick], L.mx4_dequantize(L.mx4_quantize(few)))
    del back
    turned = L.mx4_quantize(x[:, :64], transpose=True)               # blocks down columns that lie 128 KB apart
    assert torch.equal(L.mx4_dequantize(turned), L.mx4_dequantize(L.mx4_quantize(x[:, :64].contiguous(), transpose=True)))
    del turned
    y, saved = L.act8_forward("silu", x)
    y2, saved2 = L.act8_forward("silu", few)
    assert torch.equal(y[pick], y2) and torch.equal(saved.codes[pick], saved2.codes)
    used = (cols + 31) // 32
    assert torch.equal(saved.scales[pick, :used], saved2.scales[:, :used])
    dx = L.act8_backward("silu", x, saved, out=y)
    assert torch.equal(dx[pick], L.act8_backward("silu", few, saved2))
    del dx, y
    one = torch.full((rows, 8), 1.0, dtype=torch.bfloat16, device="cuda")
    dw = L.act8_weight_grad(one, saved)                              # the checkpoint's rows pass 2^32 bytes
    want = L.act8_values(saved)
    total, size = torch.zeros((2, cols), dtype=torch.float64, device="cuda")
    for r in range(0, rows, 8000):
        part = want[r:r + 8000].double()
        total += part.sum(0)
        size += part.abs().sum(0)
    assert bool(((dw[3].double() - total).abs() <= _sum_tol(rows, "f32") * size).all())
    del want, saved, q, x
    a = torch.randn((rows, 64), device="cuda")
    b = torch.randn((cols, 64), device="cuda")
    w = L.mx4_quantize(b)
    big = L.mx4_matmul(a, w)                                         # a product of 2^32 values and more
    assert torch.equal(big[pick], L.mx4_matmul(a[pick].contiguous(), w))
    del big
    t, s = torch.randn((1, cols), device="cuda").bfloat16(), L.act8_save(torch.randn((1, rows), device="cuda"))
    big = L.act8_weight_grad(t, s, torch.bfloat16)                   # cols x rows outputs
    at = torch.tensor([0, 1, 32768, 65535], device="cuda")
    assert torch.equal(big[at], L.act8_weight_grad(t[:, at].contiguous(), s, torch.bfloat16))


def test_learners_train_through_the_server():
    # weights pulled in 4 bits, products, checkpoints and gradients of all operators together: the loss of a
    # 40-class problem starts near ln 40 = 3.7 and has to fall by a quarter at least
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "learner_step.py")
    spec = importlib.util.spec_from_file_location("learner_step", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.train(updates=150)
    assert len(losses) >= 300 and np.isfinite(losses).all()
    first, last = np.mean(losses[:20]), np.mean(losses[-20:])
    assert 3.0 < first < 4.5 and last < 0.75 * first, (first, last)
