"""Sizes, constants and refusals of the learner-side operators: host code only, no GPU needed."""
import os
import re

import numpy as np
import pytest

import learner_reference as ref
from paper_1509_04210_b200 import binding as rb
from paper_1509_04210_b200 import learner

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096   # an address that is aligned and never followed: every call below is refused first


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "rudra_learner.h")).read()
    defs = {k: int(v) for k, v in re.findall(r"#define\s+(RUDRA_[A-Z0-9_]+)\s+(\d+)", text)}
    assert (defs["RUDRA_F32"], defs["RUDRA_BF16"]) == (learner.F32, learner.BF16) == (rb.GRAD_F32, rb.GRAD_BF16)
    assert {k: defs["RUDRA_ACT_" + k.upper()] for k in learner.ACTS} == learner.ACTS


@pytest.mark.parametrize("rows,cols", [(0, 0), (1, 1), (1, 32), (128, 33), (129, 128), (4096, 9216), (5, 4097), (2**31 - 128, 2**20)])
def test_sizes(rows, cols):
    L = rb.lib()
    nb = -(-cols // 32)
    assert L.rudra_mx4_codes_bytes(rows, cols) == rows * nb * 16
    assert L.rudra_mx4_scales_bytes(rows, cols) == -(-rows // 128) * -(-nb // 4) * 512
    assert L.rudra_act8_codes_bytes(rows, cols) == rows * nb * 32
    assert L.rudra_act8_scales_bytes(rows, cols) == rows * (-(-nb // 16) * 16)
    need = L.rudra_mx4_linear_workspace(rows, cols)
    assert need == 0 if rows <= 32 else need >= rows * nb * 16 + -(-rows // 128) * -(-nb // 4) * 512


def test_scale_places_are_distinct_and_fill_the_array():
    rows, nb = 300, 9
    kt = -(-nb // 4)
    r, b = np.meshgrid(np.arange(384), np.arange(4 * kt), indexing="ij")
    at = ref.mx4_scale_at(r, b, kt)
    assert sorted(at.ravel()) == list(range(rb.lib().rudra_mx4_scales_bytes(rows, nb * 32)))


def _refused(code, text):
    assert code == rb.E_INVAL and text in rb.last_error(), (code, rb.last_error())


def test_quantize_refusals():
    q = rb.lib().rudra_mx4_quantize
    _refused(q(P, 2, 4, 64, 64, 0, P, P, None), "dtype")
    _refused(q(None, 0, 4, 64, 64, 0, P, P, None), "source")
    _refused(q(P + 2, 0, 4, 64, 64, 0, P, P, None), "aligned to its elements")
    _refused(q(P, 0, 4, 64, 63, 0, P, P, None), "apart")
    _refused(q(P, 0, 2**31, 64, 64, 0, P, P, None), "RUDRA_MAX_DIM")
    _refused(q(P, 0, 4, 64, 2**62, 0, P, P, None), "ld")
    _refused(q(P, 0, 4, 64, 64, 0, P + 16, P, None), "32-byte")
    _refused(q(P, 0, 4, 64, 64, 0, P, None, None), "32-byte")
    assert q(None, 0, 0, 64, 64, 0, None, None, None) == 0 and q(None, 1, 7, 0, 0, 1, None, None, None) == 0
    d = rb.lib().rudra_mx4_dequantize
    _refused(d(P, P, 4, 64, P, 7, 64, None), "dtype")
    _refused(d(P, P + 1, 4, 64, P, 0, 64, None), "32-byte")
    _refused(d(P, P, 4, 64, None, 0, 64, None), "destination")
    assert d(None, None, 0, 64, None, 0, 64, None) == 0


def test_product_refusals():
    m = rb.lib().rudra_mx4_matmul
    _refused(m(None, P, 4, P, P, 8, 64, P, 0, 8, None), "first factor")
    _refused(m(P, P, 4, P, P + 8, 8, 64, P, 0, 8, None), "second factor")
    _refused(m(P, P, 4, P, P, 8, 64, P, 0, 7, None), "apart")
    _refused(m(P, P, 4, P, P, 8, 64, P + 1, 1, 8, None), "product")
    _refused(m(P, P, 4, P, P, 8, 2**40, P, 1, 8, None), "RUDRA_MAX_DIM")
    assert m(None, None, 0, P, P, 8, 64, None, 0, 8, None) == 0
    lin = rb.lib().rudra_mx4_linear
    need = rb.lib().rudra_mx4_linear_workspace(40, 64)
    _refused(lin(P, 0, 64, 40, P, P, 8, 64, P, 0, 8, P, need - 1, None), "workspace")
    _refused(lin(P, 0, 64, 40, P, P, 8, 64, P, 0, 8, None, need, None), "workspace")
    _refused(lin(P, 0, 64, 40, P, P, 8, 64, P, 0, 8, P + 8, need, None), "workspace")
    _refused(lin(P, 9, 64, 4, P, P, 8, 64, P, 0, 8, P, need, None), "dtype")
    _refused(lin(P, 0, 64, 4, None, P, 8, 64, P, 0, 8, P, need, None), "weights")


def test_checkpoint_refusals():
    f = rb.lib().rudra_act8_forward
    _refused(f(5, P, None, 0, 4, 64, 64, P, 64, P, P, None, None, None), "activation")
    _refused(f(-1, P, None, 0, 4, 64, 64, P, 64, P, P, None, None, None), "activation")
    _refused(f(2, P, P, 0, 4, 64, 64, P, 64, P, P, None, None, None), "second input")
    _refused(f(2, P, None, 0, 4, 64, 64, None, 64, P, P, None, None, None), "output")
    _refused(f(0, P, None, 0, 4, 64, 64, P, 64, P, P, None, None, None), "no output")
    _refused(f(4, P, P, 0, 4, 64, 64, P, 64, P, P, P, None, None), "second checkpoint")
    _refused(f(4, P, None, 0, 4, 64, 64, P, 64, P, P, P, P, None), "second input")
    b = rb.lib().rudra_act8_backward
    _refused(b(2, None, 0, 4, 64, 64, P, P, None, None, P, None, 64, None), "gradient of the output")
    _refused(b(0, P, 0, 4, 64, 64, P, P, None, None, P, None, 64, None), "no gradient")
    _refused(b(4, P, 0, 4, 64, 64, P, P, P, P, P, None, 64, None), "second input")
    _refused(b(2, P, 0, 4, 64, 64, P, P, None, None, P, P, 64, None), "second input")
    assert b(2, None, 0, 0, 64, 64, None, None, None, None, None, None, 64, None) == 0


def test_weight_gradient_refusals():
    w = rb.lib().rudra_act8_weight_grad
    need = rb.lib().rudra_act8_weight_grad_workspace
    _refused(w(P, 1, 64, 10, 64, P, P, 32, None, 0, 32, None, 0, None), "weight gradient")
    _refused(w(P, 1, 64, 10, 64, None, P, 32, P, 0, 32, None, 0, None), "checkpoint")
    _refused(w(P, 1, 63, 10, 64, P, P, 32, P, 0, 32, None, 0, None), "apart")
    _refused(w(P, 5, 64, 10, 64, P, P, 32, P, 0, 32, None, 0, None), "dtype")
    assert need(P, 1, 10, 64, 64) == 0                                   # bf16 with aligned rows needs none
    assert need(P, 9, 10, 64, 64) == 0 and need(P, 1, 2**32, 64, 64) == 0   # arguments the call refuses
    assert w(None, 1, 64, 10, 0, P, P, 32, None, 0, 32, None, 0, None) == 0


def test_pull_refusals_need_a_handle():
    assert rb.lib().rudra_ps_pull_mx4(None, 0, 1, 1, 0, P, P) == rb.E_INVAL and "handle" in rb.last_error()


def test_python_refuses_tensors_that_are_not_on_the_gpu():
    import torch

    with pytest.raises(ValueError):
        learner.mx4_quantize(torch.zeros(4, 32))
    with pytest.raises(ValueError):
        learner.mx4_quantize(torch.zeros(4))
    with pytest.raises(ValueError):
        learner.act8_forward("none", torch.zeros(4, 32))
    with pytest.raises(ValueError):
        learner.mx4_dequantize(learner.MX4(torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), 4, 32))


PROGRAM = r"""
#include <stdio.h>
#include "rudra_learner.h"

int main(void) {
  if (rudra_mx4_codes_bytes(3, 33) != 3 * 32 || rudra_act8_scales_bytes(2, 513) != 64) return 1;
  if (rudra_mx4_quantize(NULL, RUDRA_F32, 4, 64, 64, 0, NULL, NULL, NULL) != RUDRA_E_INVAL) return 2;
  if (rudra_act8_forward(RUDRA_ACT_SWIGLU + 1, NULL, NULL, RUDRA_BF16, 0, 0, 0, NULL, 0, NULL, NULL, NULL, NULL, NULL) != RUDRA_E_INVAL) return 3;
  if (rudra_ps_pull_mx4(NULL, 0, 1, 1, 0, NULL, NULL) != RUDRA_E_INVAL) return 4;
  if (rudra_mx4_quantize(NULL, RUDRA_F32, 0, 64, 64, 0, NULL, NULL, NULL) != 0) return 5;
  puts(rudra_last_error());
  return 0;
}
"""


def test_the_header_is_plain_c():
    import subprocess
    import tempfile

    lib = rb.library_path()
    rb.lib()
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "t.c"), os.path.join(d, "t")
        with open(src, "w") as f:
            f.write(PROGRAM)
        subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), src, lib,
                               "-Wl,-rpath," + os.path.dirname(lib), "-o", exe])
        out = subprocess.run([exe], capture_output=True, text=True, timeout=60)
        assert out.returncode == 0 and "handle" in out.stdout, (out.returncode, out.stdout, out.stderr)


def test_only_a_handful_of_rows_is_brought_to_mx4_inside_the_product():
    # from 17 rows on a launch of its own is the faster way, and needs the workspace for it
    need = rb.lib().rudra_mx4_linear_workspace
    assert all(need(m, k) == 0 for m in (0, 1, 8, 16) for k in (1, 4096, 9216))
    assert all(need(m, k) >= m * 16 * -(-k // 32) for m in (17, 24, 32, 33) for k in (1, 4096, 9216))
