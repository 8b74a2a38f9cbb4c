"""The products at inputs and batches that other tests leave out; 64-bit definitions and bounds as in test_gpu_learner.py."""
import numpy as np
import pytest

import learner_reference as ref
from test_gpu_learner import EPS, _check_product, _close, _dev, _learner, _normal, _np, _product, _rng, _sum_tol, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(1, 130, 320), (2, 40, 33), (7, 200, 1000), (16, 129, 96), (17, 256, 320), (32, 300, 2200), (33, 140, 320), (2305, 2049, 96)])
@pytest.mark.parametrize("dtype,pad,shift", [("f32", 0, 0), ("bf16", 0, 0), ("f32", 1, 1), ("bf16", 3, 5)])
def test_blocks_of_nan_infinity_and_zero(m, n, k, dtype, pad, shift):
    # up to 16 rows x is brought to MX4 inside the product; 2305 x 2049 goes through pairs of blocks
    L, torch = _learner(), _torch()
    x, w = _normal(m, k, 1.0, 21), _normal(n, k, 1.0, 22)
    last = m - 1
    x[last, k - 1] = np.nan                      # the last block, which is short for most k
    if m > 2:
        x[0, 0], x[1] = -np.inf, 0.0
    w[n - 1, 0], w[3, k - 1], w[5] = np.nan, np.inf, 0.0
    xd, xh = _dev(x, dtype, pad, shift)
    wd, wh = _dev(w)
    got = _np(L.mx4_matmul(xd, L.mx4_quantize(wd), torch.float32))
    a, b = ref.mx4_values(xh), ref.mx4_values(wh)
    with np.errstate(invalid="ignore"):
        want, size = _product(a, b)
    _close(got, want, k * EPS * np.where(np.isnan(size), 0.0, size))
    assert np.isnan(got[last]).all() and np.isnan(got[:, n - 1]).all() and np.isnan(got[:, 3]).all()
    if m > 2:
        assert np.isnan(got[0]).all() and (np.delete(got[1], [3, n - 1]) == 0).all() and np.isfinite(got[1, 5])


def test_rows_of_a_product_are_the_same_in_every_batch():
    # Whole numbers under one scale: every partial sum is exact in 32 bits, however the reduction is split, so rows have to
    # come out alike in batches that take x as it is (up to 16), 16, 32, 64 and 128 wide tiles, and pairs of blocks.
    L, torch = _learner(), _torch()
    n, k, rows = 2100, 2304, 2400
    gen = _rng(23)
    x = gen.choice(np.array([-6, -4, -3, -2, -1, 0, 1, 2, 3, 4, 6], dtype=np.float32), size=(rows, k))
    w = gen.choice(np.array([-6, -4, -3, -2, -1, 0, 1, 2, 3, 4, 6], dtype=np.float32), size=(n, k))
    x[:, ::32], w[:, ::32] = 4.0, 4.0            # every block's scale is 1
    xd, q = _dev(x, "bf16")[0], L.mx4_quantize(_dev(w)[0])
    want = torch.from_numpy(x).cuda().double() @ torch.from_numpy(w).cuda().double().t()
    assert float(want.abs().max()) < 2 ** 24
    for m in (1, 2, 16, 17, 32, 33, 64, 65, 100, 128, 129, 300, rows):
        assert torch.equal(L.mx4_matmul(xd[:m], q, torch.float32).double(), want[:m]), m
        assert torch.equal(L.mx4_matmul(L.mx4_quantize(xd[:m]), q, torch.float32).double(), want[:m]), m


@pytest.mark.parametrize("m", [1, 20, 33, 100, 300])
def test_rows_of_a_product_in_a_batch_and_by_themselves(m):
    # values of any size: the order of the sum may differ with the batch, its bound does not
    L, torch = _learner(), _torch()
    x, xh = _dev(_normal(m, 2000, 1.0, 24), "bf16")
    w, wh = _dev(_normal(500, 2000, 0.01, 25))
    q = L.mx4_quantize(w)
    _check_product(L.mx4_matmul(x, q, torch.float32), ref.mx4_values(xh), ref.mx4_values(wh), False)
    _check_product(L.mx4_matmul(x[m - 1:], q, torch.float32), ref.mx4_values(xh[m - 1:]), ref.mx4_values(wh), False)


@pytest.mark.parametrize("exponent", [-100, -112, -120, -126])
def test_weight_gradient_of_tiny_f32_gradients(exponent):
    # f32 gradients enter as three bf16 planes; bf16 ends at 2^-133, so that much of each gradient may be cut off
    L, torch = _learner(), _torch()
    t, n, k = 200, 40, 96
    x, xh = _dev(_normal(t, k, 2.0 ** 60, 26), "bf16")
    dy, dyh = _dev(_normal(t, n, 1.0, 27) * np.float32(2.0 ** exponent))
    got = L.act8_weight_grad(dy, L.act8_save(x))
    g, xq = dyh.astype(np.float64), ref.act8_values(xh)
    want, size = _product(np.ascontiguousarray(g.T), np.ascontiguousarray(xq.T))
    _close(_np(got), want, _sum_tol(t, "f32") * size + 2.0 ** -133 * np.abs(xq).sum(0))


def test_weight_gradient_with_infinite_and_nan_gradients():
    # an output whose gradient holds one is lost as the formula has it, the others are not
    L, torch = _learner(), _torch()
    for dtype in ("f32", "bf16"):
        x, xh = _dev(np.abs(_normal(150, 70, 1.0, 28)) + 0.5, "bf16")
        g = _normal(150, 33, 1.0, 29)
        g[140, 2], g[3, 7], g[77, 30] = np.inf, -np.inf, np.nan
        dy, dyh = _dev(g, dtype)
        got = _np(L.act8_weight_grad(dy, L.act8_save(x)))
        assert (got[2] == np.inf).all() and (got[7] == -np.inf).all() and np.isnan(got[30]).all()
        keep = [i for i in range(33) if i not in (2, 7, 30)]
        want, size = _product(np.ascontiguousarray(dyh[:, keep].astype(np.float64).T), np.ascontiguousarray(ref.act8_values(xh).T))
        _close(got[keep], want, _sum_tol(150, "f32") * size)
