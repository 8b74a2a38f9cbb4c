"""FP8 in blocks of 128 on the GPU, through the public interface: codes bit for bit, products against 64 bits.

A sum of K exact products in 32 bits is within K * 2^-23 of the sum of their magnitudes (K additions, each off by at most
one unit in the last place, truncating units included); an output in bf16 adds half a step, 2^-8 of the value."""
import numpy as np
import pytest

import block_reference as ref
from test_gpu_learner import EPS, _close, _dev, _learner, _normal, _np, _torch

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 127), (3, 128), (1, 129), (2, 511), (5, 512), (7, 513), (130, 260), (33, 1000), (129, 64), (257, 95), (64, 4096), (128, 128)]


def _check(q, x, square=False):
    codes, scales = ref.fp8_bytes(x, square)
    rows, cols = x.shape
    assert (q.rows, q.cols) == (rows, cols)
    np.testing.assert_array_equal(q.codes.cpu().numpy().reshape(codes.shape), codes)
    kt = -(-(-(-cols // 128)) // 4)
    r, b = np.meshgrid(np.arange(rows), np.arange(4 * kt), indexing="ij")
    at = ref.scale_at(r, b, kt)              # padding blocks of a row included, padding rows not
    np.testing.assert_array_equal(q.scales.cpu().numpy()[at], scales[at])


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype,pad,shift", [("f32", 0, 0), ("bf16", 0, 0), ("f32", 3, 1), ("bf16", 8, 5)])
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("square", [False, True])
def test_quantize_is_exact(rows, cols, dtype, pad, shift, transpose, square):
    L = _learner()
    x, held = _dev(_normal(rows, cols, 0.01), dtype, pad, shift)
    q = L.fp8_quantize(x, transpose, square)
    held = held.T if transpose else held
    _check(q, held, square)
    want = ref.fp8_values(held, square)
    for out in (_torch().float32, _torch().bfloat16):
        np.testing.assert_array_equal(_np(L.fp8_dequantize(q, out)), want)


def test_quantize_into_what_the_caller_has_leaves_the_rest_alone():
    torch, L = _torch(), _learner()
    x, held = _dev(_normal(37, 300))
    codes = torch.full((37 * 384 + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((512 + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    q = L.FP8(codes, scales, 37, 300)
    assert L.fp8_quantize(x, out=q) is q
    want, _ = ref.fp8_bytes(held)
    np.testing.assert_array_equal(codes[:37 * 384].cpu().numpy().reshape(37, 384), want)
    assert (codes[37 * 384:] == 0xA5).all() and (scales[512:] == 0xA5).all()
    y = torch.full((37, 310), 7.0, device="cuda")
    L.fp8_dequantize(q, out=y[:, 3:303])
    np.testing.assert_array_equal(_np(y[:, 3:303]), ref.fp8_values(held))
    assert (y[:, :3] == 7).all() and (y[:, 303:] == 7).all()


def test_ties_saturation_borders_and_signs():
    L = _learner()
    grid = np.concatenate([ref.E4M3, (ref.E4M3[1:] + ref.E4M3[:-1]) / 2])
    fine = np.concatenate([grid, np.nextafter(grid.astype(np.float32), np.float32(1e9)), np.nextafter(grid.astype(np.float32), np.float32(-1))])
    fine = fine[fine <= 448]
    row = np.zeros((len(fine) * 2, 128), dtype=np.float32)
    row[:, 0] = 448.0                     # fixes the scale at 1
    row[:, 1] = np.concatenate([fine, -fine])
    row[:, 2] = -0.0
    for scale in (1.0, 2.0 ** -100, 2.0 ** 110):
        x = (row * np.float32(scale)).astype(np.float32)
        for transpose, square in ((False, False), (True, False)):
            _check(L.fp8_quantize(_dev(x.T.copy() if transpose else x)[0], transpose, square), x, square)
    top = np.zeros((4, 128), dtype=np.float32)      # where the scale changes
    top[:, 5] = [448.0, np.nextafter(np.float32(448), np.float32(500)), 224.0, np.nextafter(np.float32(224), np.float32(0))]
    top[:, 6] = 0.3
    _check(L.fp8_quantize(_dev(top)[0]), top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("transpose,square", [(False, False), (True, False), (False, True), (True, True)])
def test_extreme_and_non_finite_blocks(dtype, transpose, square):
    L = _learner()
    x = _normal(150, 128 * 5 + 7, 1.0)
    big, tiny = np.float32(3.3895314e38), np.float32(2.0 ** -133)
    x[1, 0:128] = 0.0
    x[2, 140] = np.inf
    x[3, 270] = -np.inf
    x[4, 400] = np.nan
    x[5, 130:140] = big
    x[6, 160:192] = tiny
    x[7, 256:384] = tiny
    x[7, 293] = np.float32(2.0 ** -126)
    x[9, 384:512] = -big
    x[130:, 512:] = 0.0
    x[130, 512:] = tiny
    x[149] = np.nan
    v, held = _dev(x, dtype)
    held = held.T if transpose else held
    q = L.fp8_quantize(v, transpose, square)
    _check(q, held, square)
    # `big` is 255 * 2^120 and a little, its scale 2^120 (255 / 2^-1 > 448), and 255 lies nearer to 256 than to 240: the code
    # stands for 2^128, which a float32 holds as infinity
    with np.errstate(over="ignore"):
        want = ref.fp8_values(held, square).astype(np.float32)
    np.testing.assert_array_equal(_np(L.fp8_dequantize(q, _torch().float32)), want)


# ---------------------------------------------------------------------------------------- products

def _product(a, b, k, got, out):
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    tol = k * EPS * size + (2.0 ** -8 * np.abs(want) if out == "bf16" else 0.0) + 2.0 ** -140
    _close(got, want, np.where(np.isnan(want), 0.0, tol))      # a sum that is no number has no error: NaN on both sides


MATMULS = [(1, 1, 1), (1, 128, 128), (1, 129, 127), (2, 5, 300), (9, 200, 1000), (16, 257, 640), (17, 130, 513), (31, 64, 4096), (33, 300, 129), (64, 128, 2000),
           (65, 100, 900), (100, 1000, 1300), (128, 128, 512), (129, 257, 385), (200, 140, 2500), (300, 70, 128), (1500, 2000, 300), (1409, 1729, 513)]


@pytest.mark.parametrize("m,n,k", MATMULS)
@pytest.mark.parametrize("dtype,out,pad", [("bf16", "f32", 0), ("f32", "bf16", 3)])
def test_product(m, n, k, dtype, out, pad):
    torch, L = _torch(), _learner()
    x, held = _dev(_normal(m, k, 1.0, 1), dtype, pad, 1 if pad else 0)
    w, held_w = _dev(_normal(n, k, 0.01, 2))
    q = L.fp8_quantize(w, square=True)
    b, a = ref.fp8_values(held_w, True), ref.fp8_values(held)
    t = torch.float32 if out == "f32" else torch.bfloat16
    y = torch.full((m + 2, n + 5), 7.0, dtype=t, device="cuda")
    L.fp8_matmul(x, q, out=y[1:m + 1, 2:n + 2])
    _product(a, b, k, _np(y[1:m + 1, 2:n + 2]), out)
    assert (y[0] == 7).all() and (y[m + 1] == 7).all() and (y[:, :2] == 7).all() and (y[:, n + 2:] == 7).all()
    coded = L.fp8_matmul(L.fp8_quantize(x), q, t)      # the same codes by themselves
    assert torch.equal(coded, y[1:m + 1, 2:n + 2])


@pytest.mark.parametrize("t,n,k", [(1, 3, 5), (37, 100, 130), (509, 300, 257), (1000, 64, 1000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_a_layer(t, n, k, dtype):
    """dw = dy^T x from transposed quantizations; dx = dy w from weights whose transpose has the same values."""
    torch, L = _torch(), _learner()
    x, held_x = _dev(_normal(t, k, 1.0, 3), dtype, 3)
    dy, held_dy = _dev(_normal(t, n, 1e-3, 4), dtype)
    w, held_w = _dev(_normal(n, k, 0.02, 5))
    dw = L.fp8_matmul(L.fp8_quantize(dy, transpose=True), L.fp8_quantize(x, transpose=True), torch.float32)
    _product(ref.fp8_values(held_dy.T), ref.fp8_values(held_x.T), t, _np(dw), "f32")
    straight, turned = L.fp8_quantize(w, square=True), L.fp8_quantize(w, transpose=True, square=True)
    assert torch.equal(L.fp8_dequantize(straight, torch.float32).t(), L.fp8_dequantize(turned, torch.float32))
    _product(ref.fp8_values(held_dy), ref.fp8_values(held_w, True).T, n, _np(L.fp8_matmul(dy, turned, torch.float32)), "f32")


@pytest.mark.parametrize("m", [5, 40, 300, 1500])
def test_blocks_that_differ_by_far_and_non_finite_ones(m):
    torch, L = _torch(), _learner()
    n, k = 1500 if m == 1500 else 200, 700
    x = _normal(m, k, 1.0, 6) * np.exp2(np.repeat(np.random.default_rng(1).integers(-30, 30, (m, 6)), 128, 1)[:, :k]).astype(np.float32)
    w = _normal(n, k, 1.0, 7)
    x[1, 130] = np.inf
    x[3, 699] = np.nan
    w[7, 300] = -np.inf
    x[4] = 0.0
    (xd, held), (wd, held_w) = _dev(x.astype(np.float32)), _dev(w)
    y = _np(L.fp8_matmul(xd, L.fp8_quantize(wd), torch.float32))
    _product(ref.fp8_values(held), ref.fp8_values(held_w), k, y, "f32")
    assert np.isnan(y[1]).all() and np.isnan(y[3]).all() and np.isnan(y[:, 7]).all() and (np.delete(y[4], 7) == 0).all()


@pytest.mark.parametrize("m,n", [(1, 200), (40, 100), (300, 200), (1500, 1600)])
def test_long_sums_of_positive_values(m, n):
    """Every addition to a sum cuts it off, by 2^-23 of itself at most: a sum of s blocks of 128 values has 4 s of them, on average half
    way up, so s * 2^-22 too little at most; f32 results are gathered every 96 blocks at most, with a rounding each: under 3e-5 however long."""
    torch, L = _torch(), _learner()
    k = 60000
    a, b = torch.rand(m, k, device="cuda") + 0.5, torch.rand(n, k, device="cuda") + 0.5
    qa, qb = L.fp8_quantize(a), L.fp8_quantize(b)
    want = L.fp8_dequantize(qa, torch.float32).double() @ L.fp8_dequantize(qb, torch.float32).double().t()
    for x in (qa, a) if m <= 16 else (qa,):
        off = (L.fp8_matmul(x, qb, torch.float32).double() - want) / want
        assert off.abs().max().item() < 96 * 2.0 ** -22 + 8 * 2.0 ** -24
    off = (L.fp8_matmul(qa, qb).double() - want) / want
    assert off.abs().max().item() < 469 * 2.0 ** -22 + 2.0 ** -8


def test_empty_sizes():
    torch, L = _torch(), _learner()
    e = lambda r, c: torch.empty(r, c, device="cuda")  # noqa: E731
    assert L.fp8_matmul(e(0, 64), L.fp8_quantize(e(5, 64))).shape == (0, 5)
    assert L.fp8_matmul(e(3, 64), L.fp8_quantize(e(0, 64))).shape == (3, 0)
    y = L.fp8_matmul(e(40, 0), L.fp8_quantize(e(5, 0)), torch.float32)
    assert y.shape == (40, 5) and (y == 0).all()
    assert L.fp8_dequantize(L.fp8_quantize(e(0, 7), transpose=True)).shape == (7, 0)
    L.sync()


@pytest.mark.parametrize("m", [1, 40, 2000])
def test_a_product_does_not_depend_on_the_run(m):
    torch, L = _torch(), _learner()
    x, w = torch.randn(m, 1000, device="cuda"), L.fp8_quantize(torch.randn(1333, 1000, device="cuda"))
    first = L.fp8_matmul(x, w, torch.float32)
    assert all(torch.equal(first, L.fp8_matmul(x, w, torch.float32)) for _ in range(5))


def test_refusals():
    torch, L = _torch(), _learner()
    x, q = torch.zeros(4, 64, device="cuda"), L.fp8_quantize(torch.zeros(8, 64, device="cuda"))
    for call in (lambda: L.fp8_matmul(torch.zeros(4, 63, device="cuda"), q), lambda: L.fp8_matmul(x, x), lambda: L.fp8_matmul(x, L.mx4_quantize(x)),
                 lambda: L.mx4_matmul(x, q), lambda: L.fp8_matmul(x, q, torch.float16), lambda: L.fp8_matmul(x, q, out=torch.zeros(4, 9, device="cuda")),
                 lambda: L.fp8_quantize(x.half()), lambda: L.fp8_quantize(x.t()), lambda: L.fp8_quantize(x, out=q), lambda: L.fp8_quantize(x, out=L.mx4_quantize(x)),
                 lambda: L.fp8_matmul(x.cpu(), q), lambda: L.FP8(q.codes[:4], q.scales, 8, 64), lambda: L.fp8_dequantize(L.act8_save(x)),
                 lambda: L.fp8_matmul(x.clone().requires_grad_(), q)):
        with pytest.raises(ValueError):
            call()


def test_a_pull_has_the_servers_weights():
    torch, L = _torch(), _learner()
    from paper_1509_04210_b200 import binding as rb

    n = 300 * 200 + 50
    ps = rb.ParameterServer(n, 4, 2, 0.01, 0.9, 5e-4)
    w = _normal(1, n, 0.02, 9)[0]
    ps.set_weights(torch.from_numpy(w).cuda())
    for transpose in (False, True):
        q, ts = L.pull_fp8(ps, 13, 300, 200, transpose=transpose)
        m = w[13:13 + 60000].reshape(300, 200)
        assert ts == 0
        _check(q, m.T if transpose else m, True)
    again, _ = L.pull_fp8(ps, 13, 300, 200, transpose=True, out=q)
    assert again is q
    for bad in ((13, 300, 201), (50 + 1, 300, 200)):
        with pytest.raises(rb.RudraError):
            L.pull_fp8(ps, *bad)
    with pytest.raises(ValueError):
        L.pull_fp8(ps, 0, 300, 200, out=q)
    before = w.copy()
    ps.push(torch.ones(n, device="cuda"), 0)
    ps.push(torch.ones(n, device="cuda"), 0)
    ps.step()
    q, ts = L.pull_fp8(ps, 0, 1, n)
    slot = torch.empty(n, device="cuda")
    ps.pull(slot)
    torch.cuda.synchronize()
    assert ts == 1 and not np.array_equal(slot.cpu().numpy(), before)
    _check(q, slot.cpu().numpy().reshape(1, n), True)
