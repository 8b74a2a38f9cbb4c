"""The learner-side operators of ``include/rudra_learner.h`` on torch tensors.

Marshalling only, as in ``binding``: outputs are allocated with torch, the work runs in the native
library on torch's current stream of the inputs' device.  Matrices are two-dimensional float32 or
bfloat16 tensors whose rows are contiguous; rows may lie any distance apart.  Arguments that do not fit
raise ``ValueError`` here or ``RudraError`` from the library.  So does a tensor that requires a gradient
while torch records gradients, or has a tangent: a layer's backward pass is written out with these operators, which
record nothing themselves.  The marshalling itself is native (``csrc/learner_torch.cpp``, built on first
use if absent or stale); there is no fallback.
"""
from __future__ import annotations

import torch

from . import binding as _b
from . import build as _build

_b.lib()                      # librudra_ps.so, built first if it has to be
_build.load_learner()
from . import _learner as _n  # noqa: E402

F32, BF16 = 0, 1
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "swiglu": 4}

#: ``MX4(codes, scales, rows, cols)``: a matrix in microscaled 4-bit floating point.
MX4 = _n.MX4
#: ``Act8(codes, scales, rows, cols)``: an 8-bit checkpoint of ``rows`` tokens x ``cols`` channels.
Act8 = _n.Act8


def _act(act):
    kind = ACTS.get(act)
    if not kind:
        raise ValueError("no activation function %r" % (act,))
    return kind


def mx4_quantize(x, transpose=False, out=None):
    """``x`` in MX4, or its transpose (blocks along the columns of ``x``)."""
    return _n.mx4_quantize(x, transpose, out)


def mx4_dequantize(q, dtype=torch.bfloat16, out=None):
    """The values an MX4 matrix stands for (``dtype`` holds where ``out`` is not given, here and below)."""
    return _n.mx4_dequantize(q, dtype, out)


def mx4_matmul(a, b, dtype=torch.bfloat16, out=None):
    """``a @ b.T`` with ``b`` an MX4 matrix (rows x k) and ``a`` either one or a tensor (m x k), which is
    brought to MX4 on the way."""
    return _n.mx4_matmul(a, b, dtype, out)


def pull_mx4(ps, offset, rows, cols, transpose=False, out=None):
    """(the ``rows`` x ``cols`` matrix at weight ``offset`` of a parameter server in MX4, the weights'
    timestamp).  The work runs on the server's stream, after what torch's current stream of the server's device holds and
    before what that is given later, so the matrix is used like one that was made there."""
    m, n, device = (cols, rows, ps.device) if transpose else (rows, cols, ps.device)
    if out is None:
        out = _n.empty(0, m, n, device)
    elif not isinstance(out, MX4) or (out.rows, out.cols, out.device) != (m, n, device):
        raise ValueError("out: MX4 of %d x %d on the server's device is wanted" % (m, n))
    return out, ps.pull_mx4_on(offset, rows, cols, transpose, out.codes_ptr, out.scales_ptr, _n.current_stream(device))


def act8_save(x, out=None):
    """The 8-bit checkpoint of ``x``."""
    return _n.act8_forward(0, x, None, None, out, None)


def act8_values(saved, dtype=torch.bfloat16, out=None):
    """The values a checkpoint stands for."""
    return _n.act8_values(saved, dtype, out)


def act8_forward(act, x, up=None, out=None, saved=None, saved_up=None):
    """(f(x), checkpoint of x); for ``"swiglu"`` (silu(x) * up, checkpoint of x, checkpoint of up)."""
    return _n.act8_forward(_act(act), x, up, out, saved, saved_up)


def act8_backward(act, dy, saved, saved_up=None, out=None, out_up=None):
    """dy * f'(x) with x from its checkpoint; for ``"swiglu"`` the gradients of both inputs."""
    return _n.act8_backward(_act(act), dy, saved, saved_up, out, out_up)


def act8_weight_grad(dy, saved, dtype=torch.float32, out=None):
    """dy.T @ x with x from its checkpoint: the weight gradient of a linear layer, for instance written
    (``out``) into the layer's part of the vector that is pushed."""
    return _n.act8_weight_grad(dy, saved, dtype, out)


def sync(device=None):
    """Waits for torch's current stream; raises ``RudraError``, once on each stream, if a kernel of these operators gave up a wait
    on the device."""
    _n.synchronize(torch.cuda.current_device() if device is None else int(device))
