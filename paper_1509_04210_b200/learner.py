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


def _native():
    global _lib
    if _lib is None:
        _lib = _b.lib()
    return _lib


class MX4:
    """A matrix in microscaled 4-bit floating point: ``rows`` x ``cols``, ``codes`` and ``scales`` as the
    header lays them out (uint8 tensors)."""

    __slots__ = ("codes", "scales", "rows", "cols")

    def __init__(self, codes, scales, rows, cols):
        self.codes, self.scales, self.rows, self.cols = codes, scales, int(rows), int(cols)

    @staticmethod
    def empty(rows, cols, device="cuda"):
        nb = (cols + 31) // 32
        return MX4(torch.empty((rows, nb * 16), dtype=torch.uint8, device=device),
                   torch.empty((rows + 127) // 128 * ((nb + 3) // 4) * 512, dtype=torch.uint8, device=device), rows, cols)

    def _check(self, what):
        nb = (self.cols + 31) // 32
        _check_bytes(what, self.codes, self.rows * nb * 16)
        _check_bytes(what, self.scales, (self.rows + 127) // 128 * ((nb + 3) // 4) * 512)


class Act8:
    """An 8-bit activation checkpoint: ``tokens`` x ``channels``, int8 ``codes`` and uint8 ``scales``."""

    __slots__ = ("codes", "scales", "tokens", "channels")

    def __init__(self, codes, scales, tokens, channels):
        self.codes, self.scales, self.tokens, self.channels = codes, scales, int(tokens), int(channels)

    @staticmethod
    def empty(tokens, channels, device="cuda"):
        nb = (channels + 31) // 32
        return Act8(torch.empty((tokens, nb * 32), dtype=torch.int8, device=device),
                    torch.empty((tokens, nb), dtype=torch.uint8, device=device), tokens, channels)

    def _check(self, what):
        nb = (self.channels + 31) // 32
        _check_bytes(what, self.codes, self.tokens * nb * 32)
        _check_bytes(what, self.scales, self.tokens * nb)


def _check_bytes(what, t, nbytes):
    if not t.is_cuda or t.element_size() != 1 or not t.is_contiguous() or t.numel() < nbytes:
        raise ValueError("%s: needs %d contiguous bytes on the GPU" % (what, nbytes))


def _matrix(what, t):
    """(address, dtype, rows, cols, ld) of a matrix."""
    dtype = _DTYPES.get(t.dtype)
    if dtype is None or t.dim() != 2 or not t.is_cuda:
        raise ValueError("%s: a two-dimensional float32 or bfloat16 tensor on the GPU is wanted" % what)
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("%s: rows have to be contiguous" % what)
    return t.data_ptr(), dtype, rows, cols, ld if rows > 1 else max(ld, cols)


def _out(what, out, rows, cols, dtype, like):
    """The output given by the caller, or a new one."""
    if out is None:
        return torch.empty((rows, cols), dtype=dtype, device=like.device)
    if tuple(out.shape) != (rows, cols) or out.device != like.device or (dtype is not None and out.dtype != dtype):
        raise ValueError("%s: %d x %d of %s on the input's device is wanted" % (what, rows, cols, dtype))
    return out


def _same_device(first, *others):
    for t in others:
        if t.device != first.device:
            raise ValueError("tensors on %s and %s" % (first.device, t.device))


def _run(fn, like, *args):
    """The call on torch's current stream of the device of ``like``, with that device current."""
    device = like.device.index
    if device == torch.cuda.current_device():
        code = fn(*args, torch.cuda.current_stream().cuda_stream)
    else:
        with torch.cuda.device(device):
            code = fn(*args, torch.cuda.current_stream().cuda_stream)
    if code < 0:
        raise _b.RudraError(code, _b.last_error())


def mx4_quantize(x, transpose=False, out=None):
    """``x`` in MX4, or its transpose (blocks along the columns of ``x``)."""
    ptr, dtype, rows, cols, ld = _matrix("x", x)
    shape = (cols, rows) if transpose else (rows, cols)
    if out is None:
        out = MX4.empty(*shape, device=x.device)
    else:
        if (out.rows, out.cols) != shape:
            raise ValueError("out: %d x %d is wanted" % shape)
        out._check("out")
        _same_device(x, out.codes, out.scales)
    _run(_native().rudra_mx4_quantize, x, ptr, dtype, rows, cols, ld, int(bool(transpose)), out.codes.data_ptr(), out.scales.data_ptr())
    return out


def mx4_dequantize(q, dtype=torch.bfloat16, out=None):
    """The values an MX4 matrix stands for."""
    q._check("q")
    out = _out("out", out, q.rows, q.cols, None if out is not None else dtype, q.codes)
    ptr, kind, _, _, ld = _matrix("out", out)
    _same_device(q.codes, q.scales)
    _run(_native().rudra_mx4_dequantize, out, q.codes.data_ptr(), q.scales.data_ptr(), q.rows, q.cols, ptr, kind, ld)
    return out


def mx4_matmul(a, b, dtype=torch.bfloat16, out=None):
    """``a @ b.T`` with ``b`` an MX4 matrix (rows x k) and ``a`` either one or a tensor (m x k), which is
    brought to MX4 on the way."""
    b._check("b")
    if isinstance(a, MX4):
        a._check("a")
        m, k, like = a.rows, a.cols, a.codes
    else:
        aptr, adtype, m, k, lda = _matrix("a", a)
        like = a
    if k != b.cols:
        raise ValueError("a has rows of %d values, b of %d" % (k, b.cols))
    out = _out("out", out, m, b.rows, None if out is not None else dtype, like)
    ptr, kind, _, _, ld = _matrix("out", out)
    _same_device(like, b.codes, b.scales)
    L = _native()
    if isinstance(a, MX4):
        _same_device(like, a.scales)
        _run(L.rudra_mx4_matmul, out, a.codes.data_ptr(), a.scales.data_ptr(), m, b.codes.data_ptr(), b.scales.data_ptr(), b.rows, k,
             ptr, kind, ld)
    else:
        need = L.rudra_mx4_linear_workspace(m, k)
        work = torch.empty(need, dtype=torch.uint8, device=a.device)
        _run(L.rudra_mx4_linear, out, aptr, adtype, lda, m, b.codes.data_ptr(), b.scales.data_ptr(), b.rows, k, ptr, kind, ld,
             work.data_ptr(), need)
    return out


def pull_mx4(ps, offset, rows, cols, transpose=False, out=None):
    """(the ``rows`` x ``cols`` matrix at weight ``offset`` of a parameter server in MX4, the weights'
    timestamp); the work runs on the server's stream."""
    shape = (cols, rows) if transpose else (rows, cols)
    if out is None:
        out = MX4.empty(*shape)
    else:
        if (out.rows, out.cols) != shape:
            raise ValueError("out: %d x %d is wanted" % shape)
        out._check("out")
    return out, ps.pull_mx4(offset, rows, cols, transpose, out.codes, out.scales)


def act8_save(x, out=None):
    """The 8-bit checkpoint of ``x``."""
    return _forward("none", x, None, None, out, None)[1]


def act8_values(saved, dtype=torch.bfloat16, out=None):
    """The values a checkpoint stands for."""
    saved._check("saved")
    out = _out("out", out, saved.tokens, saved.channels, None if out is not None else dtype, saved.codes)
    ptr, kind, _, _, ld = _matrix("out", out)
    _same_device(saved.codes, saved.scales)
    _run(_native().rudra_act8_backward, out, 0, None, kind, saved.tokens, saved.channels, 0, saved.codes.data_ptr(),
         saved.scales.data_ptr(), None, None, ptr, None, ld)
    return out


def act8_forward(act, x, up=None, out=None, saved=None, saved_up=None):
    """(f(x), checkpoint of x); for ``"swiglu"`` (silu(x) * up, checkpoint of x, checkpoint of up)."""
    if act == "none":
        raise ValueError('"none" has no output: act8_save keeps a checkpoint')
    return _forward(act, x, up, out, saved, saved_up)


def _forward(act, x, up, out, saved, saved_up):
    kind = ACTS.get(act)
    if kind is None:
        raise ValueError("unknown activation %r" % (act,))
    ptr, dtype, tokens, channels, ld = _matrix("x", x)
    two = act == "swiglu"
    if two != (up is not None) or (saved_up is not None and not two):
        raise ValueError('"swiglu" alone takes a second input')
    uptr = None
    if two:
        uptr, udtype, utokens, uchannels, uld = _matrix("up", up)
        if (udtype, utokens, uchannels, uld) != (dtype, tokens, channels, ld):
            raise ValueError("up: the dtype, shape and row distance of x are wanted")
    yptr, ldy, y = None, 0, None
    if act != "none":
        y = _out("out", out, tokens, channels, x.dtype, x)
        yptr, _, _, _, ldy = _matrix("out", y)
    saved = _checkpoint("saved", saved, tokens, channels, x)
    if two:
        saved_up = _checkpoint("saved_up", saved_up, tokens, channels, x)
        _same_device(x, up)
    _run(_native().rudra_act8_forward, x, kind, ptr, uptr, dtype, tokens, channels, ld, yptr, ldy, saved.codes.data_ptr(),
         saved.scales.data_ptr(), saved_up.codes.data_ptr() if two else None, saved_up.scales.data_ptr() if two else None)
    return (y, saved, saved_up) if two else (y, saved)


def _checkpoint(what, saved, tokens, channels, like):
    if saved is None:
        return Act8.empty(tokens, channels, device=like.device)
    if (saved.tokens, saved.channels) != (tokens, channels):
        raise ValueError("%s: a checkpoint of %d x %d is wanted" % (what, tokens, channels))
    saved._check(what)
    _same_device(like, saved.codes, saved.scales)
    return saved


def act8_backward(act, dy, saved, saved_up=None, out=None, out_up=None):
    """dy * f'(x) with x from its checkpoint; for ``"swiglu"`` the gradients of both inputs."""
    kind = ACTS.get(act)
    if not kind:
        raise ValueError("no activation %r with a gradient" % (act,))
    two = act == "swiglu"
    if two != (saved_up is not None) or (out_up is not None and not two):
        raise ValueError('"swiglu" alone has a second checkpoint')
    ptr, dtype, tokens, channels, ld = _matrix("dy", dy)
    saved = _checkpoint("saved", saved, tokens, channels, dy)
    dx = _out("out", out, tokens, channels, dy.dtype, dy)
    xptr, _, _, _, ldx = _matrix("out", dx)
    dup = dptr = None
    if two:
        saved_up = _checkpoint("saved_up", saved_up, tokens, channels, dy)
        dup = _out("out_up", out_up, tokens, channels, dy.dtype, dy)
        dptr, _, _, _, ldup = _matrix("out_up", dup)
        if ldup != ldx:
            raise ValueError("out_up: the row distance of out is wanted")
    _run(_native().rudra_act8_backward, dy, kind, ptr, dtype, tokens, channels, ld, saved.codes.data_ptr(), saved.scales.data_ptr(),
         saved_up.codes.data_ptr() if two else None, saved_up.scales.data_ptr() if two else None, xptr, dptr, ldx)
    return (dx, dup) if two else dx


def act8_weight_grad(dy, saved, dtype=torch.float32, out=None):
    """dy.T @ x with x from its checkpoint: the weight gradient of a linear layer, for instance written
    (``out``) into the layer's part of the vector that is pushed."""
    ptr, kind, tokens, n, ld = _matrix("dy", dy)
    if saved.tokens != tokens:
        raise ValueError("dy has %d tokens, the checkpoint %d" % (tokens, saved.tokens))
    saved._check("saved")
    _same_device(dy, saved.codes, saved.scales)
    out = _out("out", out, n, saved.channels, None if out is not None else dtype, dy)
    wptr, wkind, _, _, ldw = _matrix("out", out)
    L = _native()
    need = L.rudra_act8_weight_grad_workspace(ptr, kind, tokens, n, ld)
    work = torch.empty(need, dtype=torch.uint8, device=dy.device) if need else None
    _run(L.rudra_act8_weight_grad, dy, ptr, kind, ld, tokens, n, saved.codes.data_ptr(), saved.scales.data_ptr(), saved.channels,
         wptr, wkind, ldw, work.data_ptr() if need else None, need)
    return out
