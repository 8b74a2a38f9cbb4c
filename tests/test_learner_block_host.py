"""Sizes, refusals and sources of the 8-bit product, the norm and the clipping: no GPU needed."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import block_reference as ref
from paper_1509_04210_b200 import binding as rb
from paper_1509_04210_b200 import learner

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1509_04210_b200", "csrc")
P = 4096   # an address that is aligned and never followed: every call below is refused first


def _refused(code, text):
    assert code == rb.E_INVAL and text in rb.last_error(), (code, rb.last_error())


@pytest.mark.parametrize("rows,cols", [(0, 0), (1, 1), (1, 128), (128, 129), (129, 512), (4096, 9216), (5, 4097), (2**31 - 128, 2**20)])
def test_sizes(rows, cols):
    L = rb.lib()
    nb = -(-cols // 128)
    assert L.rudra_fp8_codes_bytes(rows, cols) == rows * nb * 128
    assert L.rudra_fp8_scales_bytes(rows, cols) == -(-rows // 128) * -(-nb // 4) * 512
    need = L.rudra_fp8_linear_workspace(rows, cols)
    assert need == 0 if rows <= 16 else need >= rows * nb * 128 + -(-rows // 128) * -(-nb // 4) * 512
    assert (L.rudra_rms_norm_backward_workspace(rows, cols) > 0) <= (rows > 0 and cols > 0)
    assert L.rudra_grad_norm_workspace(rows) >= 8


def test_fp8_refusals():
    L = rb.lib()
    q = L.rudra_fp8_quantize
    _refused(q(P, 2, 4, 64, 64, 0, 0, P, P, None), "dtype")
    _refused(q(None, 0, 4, 64, 64, 0, 0, P, P, None), "source")
    _refused(q(P + 1, 1, 4, 64, 64, 0, 0, P, P, None), "aligned to its elements")
    _refused(q(P, 0, 4, 64, 63, 0, 1, P, P, None), "apart")
    _refused(q(P, 0, 2**31, 64, 64, 1, 0, P, P, None), "RUDRA_MAX_DIM")
    _refused(q(P, 0, 4, 64, 64, 0, 0, P + 16, P, None), "32-byte")
    assert q(None, 0, 0, 64, 64, 0, 0, None, None, None) == 0 and q(None, 1, 7, 0, 0, 1, 1, None, None, None) == 0
    d = L.rudra_fp8_dequantize
    _refused(d(P, P, 4, 64, P, 7, 64, None), "dtype")
    _refused(d(P, P + 1, 4, 64, P, 0, 64, None), "32-byte")
    _refused(d(P, P, 4, 64, None, 0, 64, None), "destination")
    m = L.rudra_fp8_matmul
    _refused(m(None, P, 4, P, P, 8, 64, P, 0, 8, None), "first factor")
    _refused(m(P, P, 4, P, P + 8, 8, 64, P, 0, 8, None), "second factor")
    _refused(m(P, P, 4, P, P, 8, 64, P, 0, 7, None), "apart")
    _refused(m(P, P, 4, P, P, 8, 2**40, P, 1, 8, None), "RUDRA_MAX_DIM")
    lin, need = L.rudra_fp8_linear, L.rudra_fp8_linear_workspace(40, 64)
    _refused(lin(P, 0, 64, 40, P, P, 8, 64, P, 0, 8, P, need - 1, None), "workspace")
    _refused(lin(P, 0, 64, 40, P, P, 8, 64, P, 0, 8, P + 8, need, None), "workspace")
    _refused(lin(P, 0, 64, 4, None, P, 8, 64, P, 0, 8, None, 0, None), "weights")
    for pull, more in ((L.rudra_ps_pull_fp8, ()), (L.rudra_ps_pull_fp8_on, (None,))):
        assert pull(None, 0, 1, 1, 0, P, P, *more) == rb.E_INVAL and "handle" in rb.last_error()


def test_norm_refusals():
    L = rb.lib()

    def f(x=P, ldx=64, r=None, ldr=64, dtype=0, t=4, c=64, w=P, wt=0, eps=1e-6, s=None, lds=64, y=P, ldy=64, q=None, qs=None, a=None, as_=None):
        return L.rudra_rms_norm(x, ldx, r, ldr, dtype, t, c, w, wt, eps, s, lds, y, ldy, q, qs, a, as_, None)

    _refused(f(dtype=5), "dtype")
    _refused(f(x=None), "input")
    _refused(f(ldx=63), "apart")
    _refused(f(w=None), "weight")
    _refused(f(w=P + 1, wt=1), "weight")
    _refused(f(wt=3), "weight")
    _refused(f(r=P), "go together")
    _refused(f(s=P), "go together")
    _refused(f(r=P, s=P, ldr=5), "residual")
    _refused(f(r=P, s=P, lds=5), "sum")
    _refused(f(y=P + 2), "output")
    _refused(f(r=P, s=2 * P, y=2 * P), "one matrix")
    _refused(f(y=None), "no output")
    _refused(f(q=P), "FP8")
    _refused(f(q=P, qs=P + 8), "FP8")
    _refused(f(a=P), "checkpoint")
    for eps in (-1.0, float("nan"), float("inf")):
        _refused(f(eps=eps), "eps")
    assert f(x=None, t=0, w=None, y=None) == 0

    def b(dy=P, s=P, m=None, dtype=1, t=400, c=64, w=P, wt=0, eps=1e-6, ds=P, ldds=64, dw=P, dwt=0, ws=P, n=1 << 30):
        return L.rudra_rms_norm_backward(dy, 64, s, 64, m, 64, dtype, t, c, w, wt, eps, ds, ldds, dw, dwt, ws, n, None)

    _refused(b(dy=None), "gradient of the output")
    _refused(b(s=P + 1), "normed input")
    _refused(b(m=P + 1), "gradient of the sum")
    _refused(b(w=None), "weight")
    _refused(b(ds=None), "gradient of the input")
    _refused(b(ldds=1), "apart")
    _refused(b(dw=None), "weight gradient")
    _refused(b(dw=P + 2), "weight gradient")
    _refused(b(dwt=9), "dtype")
    _refused(b(ws=None), "workspace")
    _refused(b(ws=P + 4), "workspace")
    _refused(b(n=L.rudra_rms_norm_backward_workspace(400, 64) - 1), "workspace")
    _refused(b(eps=float("nan")), "eps")


def _list(*grads):
    """(pointers, dtypes, sizes, count) of (address, dtype, size)."""
    n = len(grads)
    return (C.c_void_p * n)(*[g[0] for g in grads]), (C.c_int * n)(*[g[1] for g in grads]), (C.c_uint64 * n)(*[g[2] for g in grads]), n


def test_clipping_refusals():
    L = rb.lib()
    need = L.rudra_grad_norm_workspace(1)
    one = _list((P, 0, 10))
    _refused(L.rudra_grad_norm(None, None, None, 1, P, P, need, None), "null")
    _refused(L.rudra_grad_norm(*one, None, P, need, None), "norm")
    _refused(L.rudra_grad_norm(*one, P + 2, P, need, None), "norm")
    _refused(L.rudra_grad_norm(*one, P, P, need - 1, None), "workspace")
    _refused(L.rudra_grad_norm(*one, P, P + 8, need, None), "workspace")
    _refused(L.rudra_grad_norm(*_list((P, 4, 10)), P, P, need, None), "dtype")
    _refused(L.rudra_grad_norm(*_list((P + 2, 0, 10)), P, P, need, None), "gradient 0")
    _refused(L.rudra_grad_norm(*_list((P, 0, 10), (None, 1, 1)), P, P, need, None), "gradient 1")
    _refused(L.rudra_grad_norm(*_list((P, 0, 2**43 + 1)), P, P, need, None), "2^43")
    _refused(L.rudra_grad_norm(*_list((P, 0, 2**42), (P, 0, 2**42 + 1)), P, P, need, None), "2^43")

    def clip(grads, outs, max_norm=1.0):
        g, t, n, count = _list(*grads)
        o = (C.c_void_p * count)(*[v[0] for v in outs])
        return L.rudra_grad_clip(g, t, n, count, P, 0, max_norm, o, (C.c_int * count)(*[v[1] for v in outs]), P, 1 << 30, None)

    _refused(L.rudra_grad_clip(*one, P, 1, 1.0, None, None, None, 0, None), "null")
    o, d = (C.c_void_p * 1)(P), (C.c_int * 1)(0)
    for known, at, n in ((0, None, need), (0, P, need - 1), (0, P + 4, need)):
        _refused(L.rudra_grad_clip(*one, P, known, 1.0, o, d, at, n, None), "workspace")
    _refused(L.rudra_grad_clip(*one, None, 1, 1.0, o, d, None, 0, None), "norm")
    _refused(clip([(P, 0, 10)], [(P, 0)], -1.0), "max_norm")
    _refused(clip([(P, 0, 10)], [(P, 0)], float("nan")), "max_norm")
    _refused(clip([(P, 0, 10)], [(P + 1, 1)]), "gradient 0")
    Q = 1 << 20
    for grads, outs in (([(P, 0, 10)], [(P, 1)]), ([(P, 0, 10)], [(P + 4, 0)]), ([(P, 0, 10), (P + 36, 0, 5)], [(Q, 0), (Q + 36, 0)]), ([(P, 0, 10), (Q, 0, 10)], [(Q, 0), (P, 0)]),
                        ([(P, 0, 10), (P, 0, 10)], [(P, 0), (P, 0)]), ([(P, 0, 10), (P + 36, 0, 10)], [(P, 0), (P + 36, 0)]), ([(P, 0, 10), (P + 60, 1, 10)], [(Q, 0), (P + 20, 1)])):
        _refused(clip(grads, outs), "overlap")
    _refused(clip([(Q, 0, 4096)], [(P - 64, 0)]), "overlap")      # the norm is at P
    _refused(clip([(P - 36, 0, 10)], [(Q, 0)]), "overlap")        # in a gradient's last value, and in its first
    _refused(clip([(Q, 0, 10), (P, 1, 10)], [(2 * Q, 0), (3 * Q, 1)]), "overlap")


def test_tensors_that_are_refused_without_a_gpu():
    x, w = torch.zeros(4, 32), torch.ones(32)
    for call in (lambda: learner.fp8_quantize(x), lambda: learner.rms_norm(x, w), lambda: learner.rms_norm_backward(x, x, w), lambda: learner.grad_norm([x]),
                 lambda: learner.clip_gradients([x], 1.0), lambda: learner.fp8_matmul(x, x), lambda: learner.FP8(torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 4, 128)):
        with pytest.raises(ValueError):
            call()
    r = torch.zeros(4, 32, requires_grad=True)
    for call in (lambda: learner.fp8_quantize(r), lambda: learner.rms_norm(r, w), lambda: learner.rms_norm_backward(x, r, w), lambda: learner.grad_norm([r])):
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="on the GPU"):
            call()
    for call in (lambda: learner.grad_norm([]), lambda: learner.clip_gradients((), 1.0)):
        with pytest.raises(ValueError, match="empty"):
            call()
    for call in (lambda: learner.grad_norm(3), lambda: learner.clip_gradients([x], "much")):
        with pytest.raises((TypeError, ValueError)):
            call()


class _Codes:
    """In the place of an FP8 matrix."""

    def __init__(self, rows, cols, device):
        self.rows, self.cols, self.device, self.codes_ptr, self.scales_ptr = rows, cols, device, 4096, 8192


class _Server:
    device = 3

    def __init__(self):
        self.calls = []

    def pull_fp8_on(self, *args):
        self.calls.append(args)
        return 17


@pytest.mark.parametrize("transpose", [False, True])
def test_a_pull_lies_on_the_servers_device_and_between_the_work_of_torchs_stream(monkeypatch, transpose):
    made = []

    def empty(kind, rows, cols, device):
        assert kind == 2
        made.append(_Codes(rows, cols, device))
        return made[-1]

    monkeypatch.setattr(learner, "FP8", _Codes)
    monkeypatch.setattr(learner._n, "empty", empty)
    monkeypatch.setattr(learner._n, "current_stream", lambda device: 1000 + device)
    ps = _Server()
    q, ts = learner.pull_fp8(ps, 7, 5, 40, transpose=transpose)
    assert ts == 17 and made == [q] and (q.rows, q.cols, q.device) == ((40, 5, 3) if transpose else (5, 40, 3))
    assert ps.calls == [(7, 5, 40, transpose, 4096, 8192, 1003)]
    for bad in (_Codes(9, 40, 3), _Codes(q.rows, q.cols, 0), object()):
        with pytest.raises(ValueError):
            learner.pull_fp8(ps, 7, 5, 40, transpose=transpose, out=bad)


def test_the_definition_of_the_backward_pass_agrees_with_differences():
    rng = np.random.default_rng(3)
    s, w, g = rng.standard_normal((5, 40)), 1 + 0.2 * rng.standard_normal(40), rng.standard_normal((5, 40))
    ds, dw, _, _ = ref.norm_backward(g, s, w, 1e-6)
    h = 1e-5
    for i, j in ((0, 0), (3, 17), (4, 39)):
        e = np.zeros_like(s)
        e[i, j] = h
        d = ((ref.norm(s + e, w, 1e-6) - ref.norm(s - e, w, 1e-6)) * g).sum() / (2 * h)
        assert abs(d - ds[i, j]) < 1e-8
        d = ((ref.norm(s, w + e[i], 1e-6) - ref.norm(s, w - e[i], 1e-6)) * g).sum() / (2 * h)
        assert abs(d - dw[j]) < 1e-8


def test_the_definition_of_fp8():
    assert len(ref.E4M3) == 127 and ref.E4M3[-1] == 448 and (np.diff(ref.E4M3) > 0).all()
    t = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(t, ref.E4M3)


# ---------------------------------------------------------------------------------------- sources

FILES = ["fp8.cu", "fp8_matmul.cu", "fp8_matmul_pair.cu", "grad_clip.cu", "rms_norm.cu"]


def _code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def test_kernels_that_overlap_with_the_one_before_are_known():
    assert sorted(f for f in os.listdir(CSRC) if f.endswith(".cu") and "launch_overlapped(" in _code(f)) == FILES
    assert all("<<<" not in _code(f) for f in FILES)


@pytest.mark.parametrize("name", FILES + ["fp8.cuh"])
def test_what_the_kernel_before_writes_is_not_read_as_read_only(name):
    code = _code(name)
    assert not re.findall(r"__ldg\b|__ldcs\b|__ldcg\b|__ldca\b|__restrict__|ld\.global\.nc", code)
    for asm in re.findall(r"asm[^;]*?\"[^;]*?ld\.global.*?;\s*(?=\n)", code, flags=re.S):
        assert "volatile" in asm[:20] and '"memory"' in asm, asm


@pytest.mark.parametrize("name", FILES)
def test_every_kernel_waits_for_the_one_before(name):
    code = _code(name)
    kernels = len(re.findall(r"__global__", code))
    assert kernels and kernels == code.count("await_previous_kernel();") == code.count("admit_next_kernel();")


@pytest.mark.parametrize("name", ["fp8_matmul.cu", "fp8_matmul_pair.cu", "rms_norm.cu"])
def test_products_and_rings_wait_as_whole_warps_and_end_with_their_copies_landed(name):
    code = _code(name)
    assert "barrier_try(" not in code and "multicast" not in code
    ends = re.findall(r"[^\n]*\bawait_copies\(", code)
    assert len(ends) == code.count("barrier_expect(") == 1
    assert re.fullmatch(r"\s*(if \(rank == 0\) )?await_copies\(", ends[0])


def test_all_counts_of_given_up_waits_are_reported():
    text = open(os.path.join(CSRC, "learner.cu")).read()
    body = text[text.index("int rudra_learner_sync("):]
    files = [f for f in sorted(os.listdir(CSRC)) if f.endswith(".cu") and "g_gave_up;" in _code(f)]
    assert len(files) == len(re.findall(r"_gave_up\(&counts\[\d\], stream\)", body)) == int(re.search(r"kKernels = (\d+)", _code("reports.h")).group(1))


PROGRAM = r"""
#include <stdio.h>
#include "rudra_learner.h"

int main(void) {
  if (rudra_fp8_codes_bytes(3, 129) != 3 * 256 || rudra_fp8_scales_bytes(129, 513) != 2 * 2 * 512) return 1;
  if (rudra_fp8_quantize(NULL, RUDRA_F32, 4, 64, 64, 0, 1, NULL, NULL, NULL) != RUDRA_E_INVAL) return 2;
  if (rudra_rms_norm(NULL, 0, NULL, 0, RUDRA_BF16, 0, 0, NULL, RUDRA_F32, 1e-6f, NULL, 0, NULL, 0, NULL, NULL, NULL, NULL, NULL) != 0) return 3;
  if (rudra_grad_clip(NULL, NULL, NULL, 1, NULL, 0, 1.0f, NULL, NULL, NULL, 0, NULL) != RUDRA_E_INVAL) return 4;
  if (rudra_ps_pull_fp8(NULL, 0, 1, 1, 0, NULL, NULL) != RUDRA_E_INVAL) return 5;
  return 0;
}
"""


def test_the_header_is_plain_c(tmp_path):
    import subprocess

    lib = rb.library_path()
    rb.lib()
    (tmp_path / "t.c").write_text(PROGRAM)
    exe = str(tmp_path / "t")
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(tmp_path / "t.c"), lib,
                           "-Wl,-rpath," + os.path.dirname(lib), "-o", exe])
    assert subprocess.run([exe], timeout=60).returncode == 0
