"""The norm of many bf16 rows, through rings of every shape that the sizes lead to, on the GPU against 64 bits; the bounds are
derived in test_gpu_norm.py."""
import pytest

from test_gpu_learner import _learner, _torch

pytestmark = pytest.mark.gpu
U, EPS = 2.0 ** -24, 1e-6

#: (rows, columns): widths of every number of warps to a row; rows enough for three to a group of every SM, and some more.
#: (test_norm_rows.py holds these to be all shapes that there are.)
RINGS = [(10_669, 504), (10_700, 40), (10_661, 264), (7_117, 1000), (7_109, 856), (3_557, 1464), (3_560, 1928), (2_233, 2520), (2_231, 2960), (1_781, 3464), (1_791, 4096), (1_345, 4496), (1_339, 5000),
         (901, 5624), (889, 6000), (893, 6656), (891, 7032), (899, 7680), (903, 8056), (447, 8704), (450, 9216), (445, 9728), (449, 10_232), (463, 10_600), (446, 11_008), (453, 11_776), (455, 12_280), (451, 12_296),
         (448, 13_832), (457, 14_400), (445, 16_384)]


def _near(got, want, tol, what):
    off = (got.double() - want).abs() - tol
    assert not off.isnan().any() and (off <= 0).all(), "%s: past its bound by %.3g" % (what, off.max().item())


def _block_tops(v, block):
    """The largest magnitude of every value's block."""
    torch = _torch()
    t, c = v.shape
    m = torch.nn.functional.pad(v.abs(), (0, -c % block)).view(t, -1, block).amax(2)
    return m.repeat_interleave(block, 1)[:, :c]


@pytest.mark.parametrize("t,c", RINGS)
@pytest.mark.parametrize("pad", [0, 8])
def test_rings(t, c, pad):
    torch, L = _torch(), _learner()
    gen = torch.Generator("cuda").manual_seed(c + pad)
    mk = lambda std: (torch.randn(t, c + pad, device="cuda", generator=gen) * std).bfloat16()[:, :c]  # noqa: E731
    x, r, dy, more = mk(0.7), mk(2.0), mk(1e-3), mk(1e-3)
    w = 1.0 + 0.2 * torch.randn(c, device="cuda", generator=gen)
    wd, tol = w.double(), (32 + c / 8192) * U
    for residual in (r, None):
        s = x if residual is None else (x.double() + r.double()).float().bfloat16()
        v = s.double()
        inv = (v.pow(2).mean(1, keepdim=True) + EPS).rsqrt()
        want = v * inv * wd
        out = torch.full((t, c + pad), 7.0, dtype=torch.bfloat16, device="cuda")
        got = L.rms_norm(x, w, residual, eps=EPS, out=out[:, :c])
        if residual is not None:
            got, total = got
            assert torch.equal(total, s)
        _near(got, want, tol * want.abs() * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs(), "y")
        assert (out[:, c:] == 7).all()
        made = L.rms_norm(x, w, residual, eps=EPS, fp8=True, keep=True)
        y8, kept = made[0], made[-1]
        top = _block_tops(want, 128)
        _near(L.fp8_dequantize(y8, torch.float32), want, torch.maximum(want.abs() * (1 + tol) / 16, top / 224 * (1 + 2 * tol) * 2.0 ** -10) + tol * want.abs() + 2.0 ** -149, "FP8")
        top = _block_tops(want, 32)
        _near(L.act8_values(kept, torch.float32), want, top / 127 * (1 + tol) + tol * top + 2.0 ** -149, "ACT8")
        assert residual is None or torch.equal(made[1], s)
    s = x.contiguous() if pad == 0 else x
    v, g = s.double(), dy.double()
    inv = (v.pow(2).mean(1, keepdim=True) + EPS).rsqrt()
    dhat = g * wd
    plain = inv * (dhat - v * inv * inv * (dhat * v).mean(1, keepdim=True))
    size = inv * (dhat.abs() + v.abs() * inv * inv * (dhat * v).abs().mean(1, keepdim=True))
    want_w, size_w = (g * v * inv).sum(0), (g * v * inv).abs().sum(0)
    for m in (more, None):
        want, all_ = (plain, size) if m is None else (plain + m.double(), size + m.double().abs())
        ds, dw = L.rms_norm_backward(dy, s, w, eps=EPS, dsum=m)
        _near(ds, want, (96 + c / 1024) * U * all_ + 2.0 ** -8 * want.abs(), "ds")
        _near(dw, want_w, (t + 64 + c / 8192) * U * size_w, "dw")
        again = L.rms_norm_backward(dy, s, w, eps=EPS, dsum=m)
        assert torch.equal(again[0], ds) and torch.equal(again[1], dw)
    L.sync()
