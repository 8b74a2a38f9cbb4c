"""The 8-bit product, the norm and the clipping past 2^32 values and over very long rows."""
import numpy as np
import pytest

import block_reference as ref
from test_gpu_learner import EPS, _close, _learner, _np, _torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _room(gigabytes):
    torch = _torch()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip("needs %d GB of device memory" % gigabytes)


def _random(rows, cols, seed, dtype="bfloat16"):
    torch = _torch()
    x = torch.empty((rows, cols), dtype=getattr(torch, dtype), device="cuda")
    for r in range(0, rows, 1 << 16):
        x[r:r + (1 << 16)].normal_(generator=torch.Generator("cuda").manual_seed(seed + r))
    return x


def test_norm_of_many_rows():
    torch, L = _torch(), _learner()
    rows, cols = 1_100_007, 4096                # 4.5e9 values
    _room(70)
    x, r = _random(rows, cols, 1), _random(rows, cols, 2)
    w = torch.rand(cols, device="cuda") + 0.5
    pick = [0, 1, 524_287, 524_288, 1_048_576, rows - 1]
    given = [(x[i:i + 1].clone(), r[i:i + 1].clone()) for i in pick]
    y8, s, kept = L.rms_norm(x, w, r, fp8=True, keep=True, out_sum=r)
    y = L.fp8_dequantize(y8, out=x)
    for i, (a, b) in zip(pick, given):
        want = (a.float() + b.float()).bfloat16()
        assert torch.equal(s[i:i + 1], want)
        v = ref.norm(_np(want), _np(w), 1e-6)
        top = np.repeat(np.abs(v).reshape(1, -1, 128).max(axis=2), 128, axis=1)
        _close(_np(y[i:i + 1]), v, np.maximum(np.abs(v), top / 224 / 64) / 16 * 1.001 + 40 * U * np.abs(v))
    del y8, kept
    ds, dw = L.rms_norm_backward(s, s, w, out=x)    # dy = s: dw = sum of s^2 / rms
    want = torch.zeros(8, dtype=torch.float64, device="cuda")
    for at in range(0, rows, 100_000):
        part = s[at:at + 100_000].double()
        inv = (part.pow(2).mean(1, keepdim=True) + 1e-6).rsqrt()
        want += (part[:, :8].pow(2) * inv).sum(0)
    # positive terms, added over 2478 rows by a thread, then 3 groups and 148 blocks: 2640 roundings at most
    assert ((dw[:8].double() - want).abs() <= 2700 * U * want).all()
    del x, r, y, ds
    torch.cuda.empty_cache()


def test_norm_of_very_long_rows():
    torch, L = _torch(), _learner()
    for rows, cols in ((3, (1 << 24) + 5), (2, (1 << 31) - 128)):
        _room(60)
        x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
        for i in range(rows):
            x[i].normal_(generator=torch.Generator("cuda").manual_seed(i))
        w = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
        inv = [1.0 / (sum(x[i, c:c + (1 << 26)].double().pow(2).sum() for c in range(0, cols, 1 << 26)) / cols + 1e-6).sqrt() for i in range(rows)]
        y = L.rms_norm(x, w)
        # squares of a thread's pieces are added one after another: cols / 8192 of them, a rounding each, and half of that in the root
        tol = (cols / 8192 + 40) * U / 2
        for i in range(rows):
            for c in (0, 1 << 23, cols - 1000):
                v = x[i, c:c + 1000].double() * inv[i]
                assert ((y[i, c:c + 1000].double() - v).abs() <= (tol + 2.0 ** -8) * v.abs()).all()
        del x, y, w
        torch.cuda.empty_cache()


def test_quantization_and_expansion_of_many_values():
    torch, L = _torch(), _learner()
    rows, cols = 300_001, 16_500
    _room(40)
    x = _random(rows, cols, 3)
    for transpose in (False, True):
        q = L.fp8_quantize(x, transpose)
        pick = [0, 127, 128, 260_300, rows - 1] if not transpose else [0, 8191, cols - 1]
        for i in pick:
            few = L.fp8_quantize(x[i:i + 1] if not transpose else x[:, i:i + 1], transpose)
            assert torch.equal(q.codes[i:i + 1], few.codes)
        if not transpose:
            back = L.fp8_dequantize(q)
            for i in pick:
                assert torch.equal(back[i:i + 1], L.fp8_dequantize(L.fp8_quantize(x[i:i + 1])))
            del back
        del q
    del x
    torch.cuda.empty_cache()


def test_a_product_with_many_results():
    torch, L = _torch(), _learner()
    m, n, k = 600_011, 8_200, 130
    _room(30)
    a, b = L.fp8_quantize(_random(m, k, 4)), L.fp8_quantize(_random(n, k, 5))
    y = L.fp8_matmul(a, b)
    bv = _np(L.fp8_dequantize(b, torch.float32))
    rows = [0, 255, 256, 300_000, 524_288, m - 1]
    av = _np(L.fp8_dequantize(a, torch.float32)[rows])
    want = av @ bv.T
    _close(_np(y[rows]), want, k * EPS * (np.abs(av) @ np.abs(bv).T) + 2.0 ** -8 * np.abs(want))
    L.sync()
    del y, a, b
    torch.cuda.empty_cache()


def test_clipping_of_many_values():
    torch, L = _torch(), _learner()
    n = (1 << 32) + 12_345
    _room(60)
    g = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    small = torch.full((1000,), 2.0, device="cuda")
    out = torch.full((n + 1,), 7.0, device="cuda")
    norm = np.sqrt(n + 4000.0)
    got = L.clip_gradients([g, small], 10.0, out=[out[1:], small])
    assert abs(got.item() - norm) <= 6 * U * norm
    by = 10.0 / norm
    for at in (0, 1 << 31, 1 << 32, n - 4000):
        assert ((out[1 + at:1 + at + 4000].double() - by).abs() <= 8 * U * by).all()
    assert out[0] == 7 and ((small.double() - 2 * by).abs() <= 8 * U * 2 * by).all()
    lo, hi = out[1:].min().item(), out[1:].max().item()
    assert lo == hi
    del g, out
    torch.cuda.empty_cache()
