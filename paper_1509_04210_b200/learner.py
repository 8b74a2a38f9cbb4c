"""The learner-side operators of ``include/rudra_learner.h`` on torch tensors.

Marshalling only, as in ``binding``: outputs are allocated with torch, the work runs in the native
library on torch's current stream of the inputs' device.  Matrices are two-dimensional float32 or
bfloat16 tensors whose rows are contiguous; rows may lie any distance apart.  Arguments that do not fit
raise ``ValueError`` here or ``RudraError`` from the library.
"""
from __future__ import annotations

import torch

from . import binding as _b

F32, BF16 = 0, 1
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "swiglu": 4}
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}
_lib = None

_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    _current_stream = torch._C._cuda_getCurrentRawStream
else:
    def _current_stream(device):
        return torch.cuda.current_stream(device).cuda_stream


def _native():
    global _lib
    if _lib is None:
        _lib = _b.lib()
    return _lib


class _Blocks:
    """Codes and scale bytes of a matrix cut into blocks of 32, in one buffer or in two given tensors."""

    __slots__ = ("_buf", "_codes", "_scales", "_split", "codes_ptr", "scales_ptr", "device", "rows", "cols")

    def __init__(self, codes, scales, rows, cols):
        self.rows, self.cols = rows, cols = int(rows), int(cols)
        codes_bytes, scales_bytes = self._sizes(rows, cols)
        for what, t, need in (("codes", codes, codes_bytes), ("scales", scales, scales_bytes)):
            if not t.is_cuda or t.element_size() != 1 or not t.is_contiguous() or t.numel() < need:
                raise ValueError("%s of a %d x %d matrix: %d contiguous bytes on the GPU are wanted" % (what, rows, cols, need))
        self.device = codes.get_device()
        if scales.get_device() != self.device:
            raise ValueError("codes and scales on different devices")
        self._buf, self._codes, self._scales, self._split = None, codes, scales, 0
        self.codes_ptr, self.scales_ptr = codes.data_ptr(), scales.data_ptr()

    @classmethod
    def empty(cls, rows, cols, device="cuda"):
        self = cls.__new__(cls)
        self.rows, self.cols = rows, cols
        codes_bytes, scales_bytes = self._sizes(rows, cols)
        self._split = split = (codes_bytes + 511) // 512 * 512
        self._buf = buf = torch.empty(split + scales_bytes, dtype=torch.uint8, device=device)
        self._codes = self._scales = None
        self.device = buf.get_device()
        self.codes_ptr = p = buf.data_ptr()
        self.scales_ptr = p + split
        return self


class MX4(_Blocks):
    """A ``rows`` x ``cols`` matrix in microscaled 4-bit floating point; ``codes`` and ``scales`` (uint8
    tensors) as the header lays them out."""

    __slots__ = ()

    @staticmethod
    def _sizes(rows, cols):
        nb = (cols + 31) // 32
        return rows * nb * 16, (rows + 127) // 128 * ((nb + 3) // 4) * 512

    @property
    def codes(self):
        if self._codes is None:
            self._codes = self._buf[:self._sizes(self.rows, self.cols)[0]].view(self.rows, (self.cols + 31) // 32 * 16)
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            self._scales = self._buf[self._split:]
        return self._scales


class Act8(_Blocks):
    """An 8-bit checkpoint of ``rows`` tokens x ``cols`` channels: int8 ``codes``, uint8 ``scales``."""

    __slots__ = ()

    @staticmethod
    def _sizes(rows, cols):
        nb = (cols + 31) // 32
        return rows * nb * 32, rows * ((nb + 15) // 16 * 16)

    @property
    def codes(self):
        if self._codes is None:
            self._codes = self._buf[:self._sizes(self.rows, self.cols)[0]].view(torch.int8).view(self.rows, (self.cols + 31) // 32 * 32)
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            self._scales = self._buf[self._split:].view(self.rows, (self.cols + 511) // 512 * 16)
        return self._scales


def _matrix(what, t):
    """(address, dtype, rows, cols, ld) of a matrix."""
    dtype = _DTYPES.get(t.dtype)
    if dtype is None or not t.is_cuda or t.dim() != 2:
        raise ValueError("%s: a two-dimensional float32 or bfloat16 tensor on the GPU is wanted" % what)
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("%s: rows have to be contiguous" % what)
    return t.data_ptr(), dtype, rows, cols, ld if rows > 1 else max(ld, cols)


def _output(what, out, rows, cols, dtype, device):
    """(tensor, address, dtype, ld) of the output given by the caller, or of a new one."""
    if out is None:
        kind = _DTYPES.get(dtype)
        if kind is None:
            raise ValueError("%s: float32 or bfloat16 is wanted" % what)
        out = torch.empty((rows, cols), dtype=dtype, device=device)
        return out, out.data_ptr(), kind, cols
    ptr, kind, r, c, ld = _matrix(what, out)
    if (r, c) != (rows, cols) or (dtype is not None and out.dtype != dtype):
        raise ValueError("%s: a %d x %d matrix of the operator's dtype is wanted" % (what, rows, cols))
    return out, ptr, kind, ld


def _run(fn, device, others, *args):
    """The call on torch's current stream of `device`, with it current; `others`: where the other tensors are."""
    for d in others:
        if d != device:
            raise ValueError("tensors on different devices (%d and %d)" % (device, d))
    if device == _current_device():
        code = fn(*args, _current_stream(device))
    else:
        with torch.cuda.device(device):
            code = fn(*args, _current_stream(device))
    if code < 0:
        raise _b.RudraError(code, _b.last_error())


def _blocks(what, cls, given, rows, cols, device):
    """The caller's MX4 matrix or checkpoint, or a new one."""
    if given is None:
        return cls.empty(rows, cols, device=device)
    if not isinstance(given, cls) or (given.rows, given.cols) != (rows, cols):
        raise ValueError("%s: %s of %d x %d is wanted" % (what, cls.__name__, rows, cols))
    return given


def mx4_quantize(x, transpose=False, out=None):
    """``x`` in MX4, or its transpose (blocks along the columns of ``x``)."""
    ptr, dtype, rows, cols, ld = _matrix("x", x)
    out = _blocks("out", MX4, out, cols if transpose else rows, rows if transpose else cols, x.device)
    _run(_native().rudra_mx4_quantize, out.device, (x.get_device(),), ptr, dtype, rows, cols, ld, 1 if transpose else 0,
         out.codes_ptr, out.scales_ptr)
    return out


def mx4_dequantize(q, dtype=torch.bfloat16, out=None):
    """The values an MX4 matrix stands for."""
    device = q.device
    out, ptr, kind, ld = _output("out", out, q.rows, q.cols, None if out is not None else dtype, device)
    _run(_native().rudra_mx4_dequantize, device, (out.get_device(),), q.codes_ptr, q.scales_ptr, q.rows, q.cols, ptr, kind, ld)
    return out


def mx4_matmul(a, b, dtype=torch.bfloat16, out=None):
    """``a @ b.T`` with ``b`` an MX4 matrix (rows x k) and ``a`` either one or a tensor (m x k), which is
    brought to MX4 on the way."""
    device = b.device
    if isinstance(a, MX4):
        m, k, at = a.rows, a.cols, a.device
    else:
        aptr, adtype, m, k, lda = _matrix("a", a)
        at = a.get_device()
    if k != b.cols:
        raise ValueError("a has rows of %d values, b of %d" % (k, b.cols))
    out, ptr, kind, ld = _output("out", out, m, b.rows, None if out is not None else dtype, device)
    L = _native()
    if isinstance(a, MX4):
        _run(L.rudra_mx4_matmul, device, (at, out.get_device()), a.codes_ptr, a.scales_ptr, m, b.codes_ptr, b.scales_ptr, b.rows, k,
             ptr, kind, ld)
    else:
        need = L.rudra_mx4_linear_workspace(m, k)
        work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        _run(L.rudra_mx4_linear, device, (at, out.get_device()), aptr, adtype, lda, m, b.codes_ptr, b.scales_ptr, b.rows, k, ptr, kind,
             ld, work.data_ptr() if need else None, need)
    return out


def pull_mx4(ps, offset, rows, cols, transpose=False, out=None):
    """(the ``rows`` x ``cols`` matrix at weight ``offset`` of a parameter server in MX4, the weights'
    timestamp); the work runs on the server's stream."""
    out = _blocks("out", MX4, out, cols if transpose else rows, rows if transpose else cols, "cuda")
    return out, ps.pull_mx4(offset, rows, cols, transpose, out.codes_ptr, out.scales_ptr)


def act8_save(x, out=None):
    """The 8-bit checkpoint of ``x``."""
    ptr, dtype, tokens, channels, ld = _matrix("x", x)
    saved = _blocks("out", Act8, out, tokens, channels, x.device)
    _run(_native().rudra_act8_forward, saved.device, (x.get_device(),), 0, ptr, None, dtype, tokens, channels, ld, None, 0,
         saved.codes_ptr, saved.scales_ptr, None, None)
    return saved


def act8_values(saved, dtype=torch.bfloat16, out=None):
    """The values a checkpoint stands for."""
    device = saved.device
    out, ptr, kind, ld = _output("out", out, saved.rows, saved.cols, None if out is not None else dtype, device)
    _run(_native().rudra_act8_backward, device, (out.get_device(),), 0, None, kind, saved.rows, saved.cols, 0, saved.codes_ptr,
         saved.scales_ptr, None, None, ptr, None, ld)
    return out


def _act(act, second):
    kind = ACTS.get(act)
    if not kind:
        raise ValueError("no activation function %r" % (act,))
    if (act == "swiglu") != second:
        raise ValueError('"swiglu", and no other, has a second input')
    return kind


def act8_forward(act, x, up=None, out=None, saved=None, saved_up=None):
    """(f(x), checkpoint of x); for ``"swiglu"`` (silu(x) * up, checkpoint of x, checkpoint of up)."""
    kind = _act(act, up is not None)
    ptr, dtype, tokens, channels, ld = _matrix("x", x)
    device = x.get_device()
    y, yptr, _, ldy = _output("out", out, tokens, channels, x.dtype, device)
    saved = _blocks("saved", Act8, saved, tokens, channels, device)
    L = _native()
    if up is None:
        if saved_up is not None:
            raise ValueError('"swiglu", and no other, has a second checkpoint')
        _run(L.rudra_act8_forward, device, (y.get_device(), saved.device), kind, ptr, None, dtype, tokens, channels, ld, yptr, ldy,
             saved.codes_ptr, saved.scales_ptr, None, None)
        return y, saved
    uptr, udtype, utokens, uchannels, uld = _matrix("up", up)
    if (udtype, utokens, uchannels, uld) != (dtype, tokens, channels, ld):
        raise ValueError("up: the dtype, shape and row distance of x are wanted")
    saved_up = _blocks("saved_up", Act8, saved_up, tokens, channels, device)
    _run(L.rudra_act8_forward, device, (up.get_device(), y.get_device(), saved.device, saved_up.device), kind, ptr, uptr, dtype, tokens,
         channels, ld, yptr, ldy, saved.codes_ptr, saved.scales_ptr, saved_up.codes_ptr, saved_up.scales_ptr)
    return y, saved, saved_up


def act8_backward(act, dy, saved, saved_up=None, out=None, out_up=None):
    """dy * f'(x) with x from its checkpoint; for ``"swiglu"`` the gradients of both inputs."""
    kind = _act(act, saved_up is not None)
    ptr, dtype, tokens, channels, ld = _matrix("dy", dy)
    device = dy.get_device()
    if (saved.rows, saved.cols) != (tokens, channels):
        raise ValueError("saved: a checkpoint of %d x %d is wanted" % (tokens, channels))
    dx, xptr, _, ldx = _output("out", out, tokens, channels, dy.dtype, device)
    L = _native()
    if saved_up is None:
        if out_up is not None:
            raise ValueError('"swiglu", and no other, has a second gradient')
        _run(L.rudra_act8_backward, device, (saved.device, dx.get_device()), kind, ptr, dtype, tokens, channels, ld, saved.codes_ptr,
             saved.scales_ptr, None, None, xptr, None, ldx)
        return dx
    if (saved_up.rows, saved_up.cols) != (tokens, channels):
        raise ValueError("saved_up: a checkpoint of %d x %d is wanted" % (tokens, channels))
    dup, dptr, _, ldup = _output("out_up", out_up, tokens, channels, dy.dtype, device)
    if ldup != ldx:
        raise ValueError("out_up: the row distance of out is wanted")
    _run(L.rudra_act8_backward, device, (saved.device, saved_up.device, dx.get_device(), dup.get_device()), kind, ptr, dtype, tokens,
         channels, ld, saved.codes_ptr, saved.scales_ptr, saved_up.codes_ptr, saved_up.scales_ptr, xptr, dptr, ldx)
    return dx, dup


def act8_weight_grad(dy, saved, dtype=torch.float32, out=None):
    """dy.T @ x with x from its checkpoint: the weight gradient of a linear layer, for instance written
    (``out``) into the layer's part of the vector that is pushed."""
    ptr, kind, tokens, n, ld = _matrix("dy", dy)
    if saved.rows != tokens:
        raise ValueError("dy has %d tokens, the checkpoint %d" % (tokens, saved.rows))
    device = dy.get_device()
    out, wptr, wkind, ldw = _output("out", out, n, saved.cols, None if out is not None else dtype, device)
    L = _native()
    need = L.rudra_act8_weight_grad_workspace(ptr, kind, tokens, n, ld)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _run(L.rudra_act8_weight_grad, device, (saved.device, out.get_device()), ptr, kind, ld, tokens, n, saved.codes_ptr, saved.scales_ptr,
         saved.cols, wptr, wkind, ldw, work.data_ptr() if need else None, need)
    return out
