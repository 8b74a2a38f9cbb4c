"""Cases for the learner-side operators: weights in microscaled 4-bit floating point and the product
with them, 8-bit activation checkpoints and the backward pass that reads them.

``run`` makes one pass through one operator, either in plain torch operations in 32 bits (``own`` false)
or through ``paper_1509_04210_b200.learner`` (``own`` true).  ``exact`` states each operator in 64 bits.

Formats, as the library documents them:

* MX4: blocks of 32 along a row share the scale 2^(s - 127), s = max(E - 2, 0) with E the exponent field of
  the block's largest magnitude (255 for a block that holds an infinity or NaN: it stands for NaN); a value
  is an E2M1 number, nearest, ties to the even code, saturating at 6.  Two codes to a byte, low half
  first, a row's codes padded to whole blocks; the scale byte of (row r, block b) sits at
  ((r / 128) * ceil(nb / 4) + b / 4) * 512 + (r % 32) * 16 + (r % 128) / 32 * 4 + b % 4.
* ACT8: blocks of 32 along a row share the scale 2^(s - 127), s = max(E - 6, 0); a value is an integer of
  at most 127 in magnitude, nearest, ties to even.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
GELU_A, GELU_B = math.sqrt(2.0 / math.pi), 0.044715


# ---------------------------------------------------------------------------------------- cases

def _quantize(rows, cols, dtype, transpose=False, pad=0, **kw):
    return dict(op="quantize", rows=rows, cols=cols, dtype=dtype, transpose=transpose, pad=pad, **kw)


def _matmul(m, n, k, dtype, out, pad=0, **kw):
    return dict(op="matmul", m=m, n=n, k=k, dtype=dtype, out=out, pad=pad, **kw)


def _act(act, tokens, channels, dtype, pad=0, **kw):
    return dict(op="act", act=act, tokens=tokens, channels=channels, dtype=dtype, pad=pad, **kw)


def _wgrad(tokens, n, k, dtype, out, pad=0, **kw):
    return dict(op="wgrad", tokens=tokens, n=n, k=k, dtype=dtype, out=out, pad=pad, **kw)


def listed():
    return [
        # A learner receives the 9216 -> 4096 layer as a 4-bit message and expands it to work in bf16.
        _quantize(4096, 9216, "f32", name="quantize f32 4096x9216"),
        # The 1000-way layer for the backward product: blocks run along its outputs.
        _quantize(1000, 4096, "f32", transpose=True, name="quantize f32 1000x4096 T"),
        # A handful of rows of activations: the smallest call, latency counts.
        _quantize(4, 4096, "bf16", name="quantize bf16 4x4096"),
        # One row through the widest layer: answering with the trained model.
        _matmul(1, 4096, 9216, "bf16", "bf16", name="matmul 1x4096x9216"),
        # A mini-batch of 100 through the 1000-way layer, odd tile sizes, scores kept in f32.
        _matmul(100, 1000, 4096, "f32", "f32", name="matmul 100x1000x4096 f32"),
        # A learner's ordinary mini-batch in the square layer.
        _matmul(256, 4096, 4096, "bf16", "bf16", name="matmul 256x4096x4096"),
        # The largest batch in the widest layer.
        _matmul(8192, 4096, 9216, "bf16", "bf16", name="matmul 8192x4096x9216"),
        # Forward and backward of a gated activation over a large batch; gate and up are halves of one matrix.
        _act("swiglu", 8192, 4096, "bf16", name="act swiglu bf16 8192x4096"),
        # A small mini-batch in f32 with a ragged last block.
        _act("gelu", 37, 1000, "f32", name="act gelu f32 37x1000"),
        # Weight gradient of the widest layer for a mini-batch of 128, in the server's f32.
        _wgrad(128, 4096, 9216, "bf16", "f32", name="wgrad 128x4096x9216 f32"),
        # Weight gradient of the square layer for a large batch, pushed as bf16.
        _wgrad(8192, 4096, 4096, "bf16", "bf16", name="wgrad 8192x4096x4096"),
        # f32 gradients of the 1000-way layer over an odd batch.
        _wgrad(509, 1000, 4096, "f32", "f32", name="wgrad f32 509x1000x4096"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "matmul", "act", "wgrad"])
    dtype = rng.choice(["f32", "bf16"])
    pad = rng.choice([0, 0, 8, 3])
    if op == "quantize":
        return _quantize(_log(rng, 1, 4096), _log(rng, 32, 9216), dtype, rng.random() < 0.5, pad)
    if op == "matmul":
        return _matmul(_log(rng, 1, 8192), _log(rng, 32, 4096), _log(rng, 32, 9216), dtype, rng.choice(["f32", "bf16"]), pad)
    if op == "act":
        return _act(rng.choice(["relu", "silu", "gelu", "swiglu"]), _log(rng, 1, 8192), _log(rng, 32, 4096), dtype, pad)
    return _wgrad(_log(rng, 1, 8192), _log(rng, 32, 4096), _log(rng, 32, 4096), dtype, rng.choice(["f32", "bf16"]), pad)


def work(case):
    g = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": (g + 2) * n, "flops": 2 * n}                      # in; the values they stand for, as bf16
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        o = 4 if case["out"] == "f32" else 2
        return {"bytes": g * m * k + 17 * n * k // 32 + o * m * n, "flops": 2 * m * n * k}
    if case["op"] == "act":
        n = case["tokens"] * case["channels"]
        two = case["act"] == "swiglu"
        return {"bytes": (6 if two else 4) * g * n, "flops": (60 if two else 30) * n}   # x (g, u), y, dy, dx (dg, du)
    t, n, k = case["tokens"], case["n"], case["k"]
    o = 4 if case["out"] == "f32" else 2
    return {"bytes": g * t * n + 2 * t * k + o * n * k, "flops": 2 * t * n * k}


# --------------------------------------------------------------------------------------- inputs

def _normal(gen, rows, cols, std, dtype, pad):
    """rows x cols of a matrix whose rows are cols + pad long."""
    x = torch.empty(rows, cols + pad, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen)
    return x.to(dtype)[:, :cols]


def _activations(gen, rows, cols, dtype, pad):
    """Roughly normal, with a few channels an order of magnitude larger, as trained layers have them."""
    x = torch.empty(rows, cols + pad, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=gen)
    big = torch.rand(cols + pad, device="cuda", generator=gen) < 0.01
    x *= torch.where(big, 12.0, 1.0)
    return x.to(dtype)[:, :cols]


def _mx4_weights(w):
    """A matrix in the MX4 layout (codes, scales), built from its definition."""
    rows, cols = w.shape
    nb = -(-cols // 32)
    x = torch.zeros(rows, nb * 32, device=w.device)
    x[:, :cols] = w
    x = x.view(rows, nb, 32)
    e = torch.frexp(x.abs().amax(2)).exponent.to(torch.int32) - 1
    s = (e + 125).clamp(min=0)                                             # E - 2 with E = e + 127
    v = torch.ldexp(x, (127 - s).unsqueeze(2))
    step = torch.where(v.abs() < 2.0, 0.5, torch.where(v.abs() < 4.0, 1.0, 2.0))
    mag = (torch.round(v.abs() / step) * step).clamp(max=6.0)
    code = torch.bucketize(mag, torch.tensor(E2M1, device=w.device)) | torch.where(v < 0, 8, 0)
    code = code.to(torch.uint8).view(rows, nb * 32)
    codes = code[:, 0::2] | (code[:, 1::2] << 4)
    rt, kt = -(-rows // 128), -(-nb // 4)
    full = torch.zeros(rt * 128, kt * 4, dtype=torch.uint8, device=w.device)
    full[:rows, :nb] = s.to(torch.uint8)
    scales = full.view(rt, 4, 32, kt, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)
    return codes.contiguous(), scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, dtype, pad = case["op"], DTYPES[case["dtype"]], case["pad"]
    s = dict(case)
    if op == "quantize":
        s["x"] = _normal(gen, case["rows"], case["cols"], 0.01, dtype, pad)
    elif op == "matmul":
        s["x"] = _activations(gen, case["m"], case["k"], dtype, pad)
        s["codes"], s["scales"] = _mx4_weights(_normal(gen, case["n"], case["k"], 0.01, torch.float32, 0))
    elif op == "act":
        t, c = case["tokens"], case["channels"]
        if case["act"] == "swiglu":
            both = _normal(gen, t, 2 * c, 1.5, dtype, pad)
            s["x"], s["up"] = both[:, :c], both[:, c:]
        else:
            s["x"], s["up"] = _normal(gen, t, c, 1.5, dtype, pad), None
        s["dy"] = _normal(gen, t, c, 1e-3, dtype, 0)
    else:
        s["x"] = _activations(gen, case["tokens"], case["k"], torch.bfloat16, 0)
        s["dy"] = _normal(gen, case["tokens"], case["n"], 1e-3, dtype, pad)
    return s


# ---------------------------------------------------------------------------------- plain forms

def _blocks(x):
    """x in 32 bits, cut into blocks of 32 along its rows, and each block's floor(log2(max))."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -cols % 32)).view(rows, -1, 32)
    return x, torch.frexp(x.abs().amax(2, keepdim=True)).exponent - 1


def _mx4_values(x):
    """What the MX4 codes of x stand for."""
    b, e = _blocks(x)
    e = (e - 2).clamp(min=-127)
    v = torch.ldexp(b, -e).clamp(-6.0, 6.0)
    step = torch.where(v.abs() < 2.0, 0.5, torch.where(v.abs() < 4.0, 1.0, 2.0))
    return torch.ldexp(torch.round(v / step) * step, e).view(x.shape[0], -1)[:, :x.shape[1]]


def _act8_values(x):
    """What the 8-bit codes of x stand for."""
    b, e = _blocks(x)
    e = (e - 6).clamp(min=-127)
    return torch.ldexp(torch.round(torch.ldexp(b, -e)).clamp(-127.0, 127.0), e).view(x.shape[0], -1)[:, :x.shape[1]]


def _mx4_expand(codes, scales, rows, cols):
    """The values of a matrix held in the MX4 layout."""
    nb = -(-cols // 32)
    kt = -(-nb // 4)
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    v = table[torch.stack((codes & 15, codes >> 4), 2).int()].view(rows, nb, 32)
    s = scales.view(-1, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, kt * 4)[:rows, :nb]
    return torch.ldexp(v, s.int().unsqueeze(2) - 127).view(rows, nb * 32)[:, :cols]


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _act_plain(act, x):
    """f(x) and f'(x)."""
    if act == "relu":
        return torch.where(x > 0, x, torch.zeros_like(x)), (x > 0).to(x.dtype)
    if act in ("silu", "swiglu"):
        s = _sigmoid(x)
        return x * s, s * (1.0 + x * (1.0 - s))
    s = _sigmoid(2.0 * GELU_A * (x + GELU_B * x * x * x))
    return x * s, s + x * s * (1.0 - s) * 2.0 * GELU_A * (1.0 + 3.0 * GELU_B * x * x)


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    if s["op"] == "quantize":
        return _mx4_values(s["x"].t() if s["transpose"] else s["x"]).to(torch.bfloat16)
    if s["op"] == "matmul":
        w = _mx4_expand(s["codes"], s["scales"], s["n"], s["k"])
        return torch.matmul(_mx4_values(s["x"]), w.t()).to(DTYPES[s["out"]])
    if s["op"] == "act":
        dtype = s["x"].dtype
        dy, y = s["dy"].float(), _act_plain(s["act"], s["x"].float())[0]
        saved, slope = _act_plain(s["act"], _act8_values(s["x"]))
        if s["up"] is None:
            return y.to(dtype), (dy * slope).to(dtype)
        return (y * s["up"].float()).to(dtype), (dy * _act8_values(s["up"]) * slope).to(dtype), (dy * saved).to(dtype)
    return torch.matmul(s["dy"].float().t(), _act8_values(s["x"])).to(DTYPES[s["out"]])


def _run_own(s):
    from paper_1509_04210_b200 import learner

    if s["op"] == "quantize":
        return learner.mx4_dequantize(learner.mx4_quantize(s["x"], transpose=s["transpose"]), torch.bfloat16)
    if s["op"] == "matmul":
        return learner.mx4_matmul(s["x"], learner.MX4(s["codes"], s["scales"], s["n"], s["k"]), DTYPES[s["out"]])
    if s["op"] == "act":
        if s["up"] is None:
            y, saved = learner.act8_forward(s["act"], s["x"])
            return y, learner.act8_backward(s["act"], s["dy"], saved)
        y, saved, saved_up = learner.act8_forward("swiglu", s["x"], s["up"])
        return (y,) + learner.act8_backward("swiglu", s["dy"], saved, saved_up)
    return learner.act8_weight_grad(s["dy"], learner.act8_save(s["x"]), DTYPES[s["out"]])


# -------------------------------------------------------------------- the definitions in 64 bits

def _scale64(x, below):
    """Power of two of each block of 32 columns, spread over the columns; ``below``: binary places below the largest."""
    block = (torch.arange(x.shape[1], device=x.device) // 32).expand(x.shape)
    top = torch.zeros(x.shape[0], (x.shape[1] + 31) // 32, dtype=torch.float64, device=x.device)
    top = top.scatter_reduce_(1, block, x.abs(), "amax")
    p = torch.floor(torch.log2(top.clamp(min=2.0 ** -1000)))
    p = torch.where(torch.exp2(p) > top, p - 1, p)                         # log2 may round to a whole number
    p = torch.where(torch.exp2(p + 1) <= top, p + 1, p)
    return torch.exp2(torch.clamp(p - below, min=-127.0)).gather(1, block)


def _mx4_64(x):
    x = x.double()
    scale = _scale64(x, 2)
    a = x.abs() / scale
    # index of the nearest E2M1 magnitude: a midpoint belongs to the neighbour with the even index
    i = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int()
         + (a > 5.0).int())
    return torch.sign(x) * torch.tensor(E2M1, dtype=torch.float64, device=x.device)[i.long()] * scale


def _act8_64(x):
    x = x.double()
    scale = _scale64(x, 6)
    a = x.abs() / scale
    low = torch.floor(a)
    up = (a - low > 0.5) | ((a - low == 0.5) & (low % 2 == 1))
    return torch.sign(x) * torch.clamp(low + up.double(), max=127.0) * scale


def _weights64(codes, scales, rows, cols):
    r = torch.arange(rows, device=codes.device).unsqueeze(1)
    c = torch.arange(cols, device=codes.device).unsqueeze(0)
    nibble = torch.where(c % 2 == 0, codes[:, :(cols + 1) // 2].repeat_interleave(2, 1)[:, :cols] % 16,
                         codes[:, :(cols + 1) // 2].repeat_interleave(2, 1)[:, :cols] // 16).long()
    b, kt = c // 32, (cols + 127) // 128
    at = ((r // 128) * kt + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4
    mag = torch.tensor(E2M1, dtype=torch.float64, device=codes.device)[nibble % 8]
    return torch.where(nibble >= 8, -mag, mag) * torch.exp2(scales[at].double() - 127.0)


def _f64(act, x):
    """f and f' from their textbook forms."""
    if act == "relu":
        return torch.clamp(x, min=0.0), (x > 0).double()
    if act in ("silu", "swiglu"):
        half = torch.tanh(x / 2)
        return x * (1 + half) / 2, (1 + half) / 2 + x * (1 - half * half) / 4
    u = GELU_A * (x + GELU_B * x ** 3)
    t = torch.tanh(u)
    return 0.5 * x * (1 + t), 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * GELU_A * (1 + 3 * GELU_B * x * x)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        return _mx4_64(s["x"].t() if case["transpose"] else s["x"])
    if case["op"] == "matmul":
        return _mx4_64(s["x"]) @ _weights64(s["codes"], s["scales"], case["n"], case["k"]).t()
    if case["op"] == "act":
        dy, y = s["dy"].double(), _f64(case["act"], s["x"].double())[0]
        saved, slope = _f64(case["act"], _act8_64(s["x"]))
        if s["up"] is None:
            return y, dy * slope
        return y * s["up"].double(), dy * _act8_64(s["up"]) * slope, dy * saved
    return s["dy"].double().t() @ _act8_64(s["x"])
