"""Cases for the operators of a learner's residual block and of what it pushes: root-mean-square norm with the
residual's addition and an 8-bit output, its backward pass, the product in 8-bit floating point with a scale for
each block of 128, forward and as a weight gradient, and the global norm of many gradients with clipping.

``run`` makes one pass through one operator, either in plain torch operations in 32 bits (``own`` false)
or through ``paper_1509_04210_b200.learner`` (``own`` true).  ``exact`` states each operator in 64 bits.

FP8, as the library documents it: 128 consecutive values of a row (or, for weights, 128 x 128 values) share the
scale 2^(s - 127), the smallest power of two (s >= 0) under which the block's largest magnitude is at most 448; a
value is the E4M3 number nearest to x / scale, ties to the even code.  A row's codes are padded with zeros to whole
blocks; the scale byte of (row r, block b) sits at
((r / 128) * ceil(nb / 4) + b / 4) * 512 + (r % 32) * 16 + (r % 128) / 32 * 4 + b % 4.

Norm: s = x + residual, rounded to x's type; y = s * w / sqrt(mean(s^2) + eps), computed from the rounded s.
Clipping: g * min(1, max_norm / norm), norm over all gradients together.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


# ---------------------------------------------------------------------------------------- cases

def _norm(tokens, channels, dtype, weight, form, residual=True, pad=0, **kw):
    return dict(op="norm", tokens=tokens, channels=channels, dtype=dtype, weight=weight, form=form, residual=residual, pad=pad, **kw)


def _norm_backward(tokens, channels, dtype, weight, through=True, pad=0, **kw):
    return dict(op="norm_backward", tokens=tokens, channels=channels, dtype=dtype, weight=weight, through=through, pad=pad, **kw)


def _matmul(m, n, k, dtype, out, pad=0, **kw):
    return dict(op="matmul", m=m, n=n, k=k, dtype=dtype, out=out, pad=pad, **kw)


def _wgrad(tokens, n, k, dtype, out, pad=0, **kw):
    return dict(op="wgrad", tokens=tokens, n=n, k=k, dtype=dtype, out=out, pad=pad, **kw)


def _clip(count, total, dtype, out, max_norm, cut=0, **kw):
    return dict(op="clip", count=count, total=total, dtype=dtype, out=out, max_norm=max_norm, cut=cut, **kw)


def listed():
    return [
        # One token on its way into the next layer's 8-bit product: the smallest call, latency counts.
        _norm(1, 4096, "bf16", "f32", "fp8", name="norm bf16 1x4096 fp8"),
        # An odd mini-batch at the 1000-way layer's width in f32, rows a few elements apart.
        _norm(509, 1000, "f32", "f32", "plain", pad=3, name="norm f32 509x1000"),
        # The largest batch, residual stream in bf16, 8-bit output for the product that follows.
        _norm(8192, 4096, "bf16", "f32", "fp8", name="norm bf16 8192x4096 fp8"),
        # Backward pass of a small mini-batch in f32.
        _norm_backward(37, 1000, "f32", "f32", name="norm backward f32 37x1000"),
        # Backward pass of the largest batch, with the gradient that comes down the residual stream.
        _norm_backward(8192, 4096, "bf16", "f32", name="norm backward bf16 8192x4096"),
        # One row through the widest layer: answering with the trained model.
        _matmul(1, 4096, 9216, "bf16", "bf16", name="fp8 1x4096x9216"),
        # A learner's ordinary mini-batch in the square layer.
        _matmul(256, 4096, 4096, "bf16", "bf16", name="fp8 256x4096x4096"),
        # The largest batch in the widest layer.
        _matmul(8192, 4096, 9216, "bf16", "bf16", name="fp8 8192x4096x9216"),
        # Weight gradient of the 1000-way layer over an odd batch, both factors brought to 8 bits along the tokens.
        _wgrad(509, 1000, 4096, "f32", "f32", name="fp8 wgrad f32 509x1000x4096"),
        # A small model's gradients, biases among them, into the vector that is pushed.
        _clip(48, 90000, "f32", "f32", 0.1, cut=1, name="clip f32 48 of 90 thousand"),
        # Half-width gradients of a middle-sized model, pushed in the server's f32.
        _clip(301, 20_000_003, "bf16", "f32", 1.0, cut=2, name="clip bf16 301 of 20 million"),
        # The 60 965 224-weight network, layer by layer, weights and biases.
        _clip(16, 60_965_224, "f32", "f32", 1.0, name="clip f32 61 million"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "matmul", "wgrad", "clip"])
    dtype, other = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
    pad = rng.choice([0, 0, 8, 3])
    if op in ("norm", "norm_backward"):
        tokens, channels = _log(rng, 1, 8192), _log(rng, 32, 9216)
        tokens = max(1, min(tokens, 4096 * 4096 // channels))
        if op == "norm":
            return _norm(tokens, channels, dtype, other, rng.choice(["plain", "fp8"]), rng.random() < 0.7, pad)
        return _norm_backward(tokens, channels, dtype, other, rng.random() < 0.7, pad)
    if op == "matmul":
        return _matmul(_log(rng, 1, 8192), _log(rng, 32, 4096), _log(rng, 32, 9216), dtype, other, pad)
    if op == "wgrad":
        return _wgrad(_log(rng, 1, 8192), _log(rng, 32, 4096), _log(rng, 32, 4096), dtype, other, pad)
    count = _log(rng, 1, 400)
    return _clip(count, _log(rng, max(1000, 2 * count), 40_000_000), dtype, other, rng.choice([0.1, 1.0, 1000.0]), rng.randrange(1, 1 << 20))


def work(case):
    g = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        n, w = case["tokens"] * case["channels"], 4 if case["weight"] == "f32" else 2
        y = 2 if case["form"] == "fp8" else g                              # 8 bits are returned as the values they stand for
        return {"bytes": (g * (3 if case["residual"] else 1) + y) * n + w * case["channels"], "flops": 6 * n}
    if case["op"] == "norm_backward":
        n, w = case["tokens"] * case["channels"], 4 if case["weight"] == "f32" else 2
        return {"bytes": g * (4 if case["through"] else 3) * n + (w + 4) * case["channels"], "flops": 12 * n}
    o = 4 if case["out"] == "f32" else 2
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": g * m * k + n * k + o * m * n, "flops": 2 * m * n * k}
    if case["op"] == "wgrad":
        t, n, k = case["tokens"], case["n"], case["k"]
        return {"bytes": g * t * n + 2 * t * k + o * n * k, "flops": 2 * t * n * k}
    return {"bytes": (g + o) * case["total"], "flops": 3 * case["total"]}


# --------------------------------------------------------------------------------------- inputs

def _sizes(case):
    """Sizes of a list of gradients: the 60 965 224-weight network's layers, or `count` odd ones that add up to `total`."""
    if not case["cut"]:
        return [34848, 96, 307200, 256, 884736, 384, 663552, 384, 442368, 256, 9216 * 4096, 4096, 4096 * 4096, 4096, 4096 * 1000, 1000]
    rng = random.Random(case["cut"])
    share = [math.exp(rng.uniform(0.0, 7.0)) for _ in range(case["count"])]
    sizes = [max(1, int(case["total"] * v / sum(share))) for v in share]
    at = max(range(len(sizes)), key=sizes.__getitem__)
    sizes[at] += case["total"] - sum(sizes)
    return sizes


def _normal(gen, rows, cols, std, dtype, pad):
    """rows x cols of a matrix whose rows are cols + pad long."""
    x = torch.empty(rows, cols + pad, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen)
    return x.to(dtype)[:, :cols]


def _activations(gen, rows, cols, dtype, pad, std=1.0):
    """Roughly normal, with a few channels an order of magnitude larger, as trained layers have them."""
    x = torch.empty(rows, cols + pad, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen)
    big = torch.rand(cols + pad, device="cuda", generator=gen) < 0.01
    x *= torch.where(big, 12.0, 1.0)
    return x.to(dtype)[:, :cols]


def _fp8_weights(w):
    """A matrix in the FP8 layout (codes, scales) with blocks of 128 x 128, built from its definition."""
    rows, cols = w.shape
    rt, nb = -(-rows // 128), -(-cols // 128)
    x = torch.zeros(rt * 128, nb * 128, device=w.device)
    x[:rows, :cols] = w
    top = x.view(rt, 128, nb, 128).abs().amax(dim=(1, 3))
    m, e = torch.frexp(top)
    s = torch.where(top > 0, (e - 9 + (m > 0.875).int() + 127).clamp(min=0), torch.zeros_like(e))
    s = s.repeat_interleave(128, 0)                                        # a byte for each row and block
    codes = torch.ldexp(x, 127 - s.repeat_interleave(128, 1)).to(torch.float8_e4m3fn).view(torch.uint8)
    kt = -(-nb // 4)
    full = torch.zeros(rt * 128, kt * 4, dtype=torch.uint8, device=w.device)
    full[:, :nb] = s.to(torch.uint8)
    scales = full.view(rt, 4, 32, kt, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)
    return codes[:rows].contiguous(), scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, dtype = case["op"], DTYPES[case["dtype"]]
    s = dict(case)
    if op in ("norm", "norm_backward"):
        t, c, pad = case["tokens"], case["channels"], case["pad"]
        s["w"] = torch.empty(c, device="cuda").normal_(1.0, 0.2, generator=gen).to(DTYPES[case["weight"]])
        s["x"] = _activations(gen, t, c, dtype, pad, 0.7)
        if op == "norm":
            s["r"] = _activations(gen, t, c, dtype, pad, 2.0) if case["residual"] else None
        else:
            s["dy"] = _normal(gen, t, c, 1e-3, dtype, pad)
            s["ds"] = _normal(gen, t, c, 1e-3, dtype, pad) if case["through"] else None
    elif op == "matmul":
        s["x"] = _activations(gen, case["m"], case["k"], dtype, case["pad"])
        s["codes"], s["scales"] = _fp8_weights(_normal(gen, case["n"], case["k"], 0.01, torch.float32, 0))
    elif op == "wgrad":
        s["x"] = _activations(gen, case["tokens"], case["k"], torch.bfloat16, 0)
        s["dy"] = _normal(gen, case["tokens"], case["n"], 1e-3, dtype, case["pad"])
    else:
        sizes = _sizes(case)
        s["grads"] = [torch.empty(n, device="cuda").normal_(0.0, 1e-3, generator=gen).to(dtype) for n in sizes]
        s["vector"] = torch.zeros(sum(sizes), dtype=DTYPES[case["out"]], device="cuda")   # what is pushed
        s["parts"] = list(s["vector"].split(sizes))
    return s


# ---------------------------------------------------------------------------------- plain forms

def _fp8_values(x):
    """What the FP8 codes of x (a block: 128 values of a row) stand for."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -cols % 128)).view(rows, -1, 128)
    m, e = torch.frexp(b.abs().amax(2, keepdim=True))
    e = (e - 9 + (m > 0.875).int()).clamp(min=-127)
    v = torch.ldexp(b, -e)
    step = torch.frexp(v).exponent.clamp(min=-5) - 4                       # of E4M3 numbers: 2^-3 of the binade, from 2^-6 on
    v = torch.ldexp(torch.round(torch.ldexp(v, -step)), step)
    return torch.ldexp(v, e).view(rows, -1)[:, :cols]


def _fp8_expand(codes, scales, rows, cols):
    """The values of a matrix held in the FP8 layout."""
    nb = -(-cols // 128)
    kt = -(-nb // 4)
    c = codes.view(rows, nb * 128).int()
    mag, exponent = c & 7, (c >> 3) & 15
    v = torch.ldexp(torch.where(exponent > 0, mag + 8, mag).float(), exponent.clamp(min=1) - 10)
    v = torch.where(c >= 128, -v, v)
    s = scales.view(-1, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, kt * 4)[:rows, :nb]
    return torch.ldexp(v.view(rows, nb, 128), s.int().unsqueeze(2) - 127).view(rows, nb * 128)[:, :cols]


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    if s["op"] == "norm":
        x, dtype = s["x"], s["x"].dtype
        if s["r"] is not None:
            x = (x.float() + s["r"].float()).to(dtype)
        v = x.float()
        y = v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * s["w"].float()
        y = _fp8_values(y).to(torch.bfloat16) if s["form"] == "fp8" else y.to(dtype)
        return (y, x) if s["r"] is not None else (y,)
    if s["op"] == "norm_backward":
        v, dtype = s["x"].float(), s["x"].dtype
        rstd = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
        hat, dy = v * rstd, s["dy"].float()
        dhat = dy * s["w"].float()
        dx = (dhat - hat * (dhat * hat).mean(1, keepdim=True)) * rstd
        if s["ds"] is not None:
            dx = dx + s["ds"].float()
        return dx.to(dtype), (dy * hat).sum(0)
    if s["op"] == "matmul":
        w = _fp8_expand(s["codes"], s["scales"], s["n"], s["k"])
        return torch.matmul(_fp8_values(s["x"]), w.t()).to(DTYPES[s["out"]])
    if s["op"] == "wgrad":
        return torch.matmul(_fp8_values(s["dy"].t()), _fp8_values(s["x"].t()).t()).to(DTYPES[s["out"]])
    norm = torch.stack([(g.float() * g.float()).sum() for g in s["grads"]]).sum().sqrt()
    c = (s["max_norm"] / norm).clamp(max=1.0)
    return norm, torch.cat([(g.float() * c).to(s["vector"].dtype) for g in s["grads"]])


def _run_own(s):
    from paper_1509_04210_b200 import learner

    if s["op"] == "norm":
        got = learner.rms_norm(s["x"], s["w"], residual=s["r"], eps=EPS, fp8=s["form"] == "fp8")
        y, more = (got[0], got[1:]) if s["r"] is not None else (got, ())
        return (learner.fp8_dequantize(y, torch.bfloat16) if s["form"] == "fp8" else y,) + more
    if s["op"] == "norm_backward":
        return learner.rms_norm_backward(s["dy"], s["x"], s["w"], eps=EPS, dsum=s["ds"])
    if s["op"] == "matmul":
        return learner.fp8_matmul(s["x"], learner.FP8(s["codes"], s["scales"], s["n"], s["k"]), DTYPES[s["out"]])
    if s["op"] == "wgrad":
        return learner.fp8_matmul(learner.fp8_quantize(s["dy"], transpose=True), learner.fp8_quantize(s["x"], transpose=True), DTYPES[s["out"]])
    return learner.clip_gradients(s["grads"], s["max_norm"], out=s["parts"]), s["vector"]


# -------------------------------------------------------------------- the definitions in 64 bits

def _e4m3_table(device):
    """The non-negative E4M3 numbers in the order of their codes."""
    values = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)]
    return torch.tensor(values, dtype=torch.float64, device=device)


def _fp8_64(x):
    x = x.double()
    block = (torch.arange(x.shape[1], device=x.device) // 128).expand(x.shape)
    top = torch.zeros(x.shape[0], (x.shape[1] + 127) // 128, dtype=torch.float64, device=x.device)
    top = top.scatter_reduce_(1, block, x.abs(), "amax")
    p = torch.ceil(torch.log2((top / 448.0).clamp(min=2.0 ** -1000)))
    p = torch.where(448.0 * torch.exp2(p) < top, p + 1, p)                 # log2 may round to a whole number
    p = torch.where(448.0 * torch.exp2(p - 1) >= top, p - 1, p)
    scale = torch.exp2(p.clamp(min=-127.0)).gather(1, block)
    table = _e4m3_table(x.device)
    a = x.abs() / scale
    # the code below a, or the one above past the midpoint; a midpoint belongs to the even one
    low = (torch.searchsorted(table, a.contiguous(), right=True) - 1).clamp(max=len(table) - 2)
    mid = (table[low] + table[low + 1]) / 2
    code = low + ((a > mid) | ((a == mid) & (low % 2 == 1))).long()
    return torch.sign(x) * table[code] * scale


def _weights64(codes, scales, rows, cols):
    r = torch.arange(rows, device=codes.device).unsqueeze(1)
    c = torch.arange(cols, device=codes.device).unsqueeze(0)
    code = codes[:, :cols].long()
    b, kt = c // 128, (cols + 511) // 512
    at = ((r // 128) * kt + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4
    mag = _e4m3_table(codes.device)[code % 128]
    return torch.where(code >= 128, -mag, mag) * torch.exp2(scales[at].double() - 127.0)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "norm_backward"):
        x, w = s["x"].double(), s["w"].double()
        if case["op"] == "norm" and s["r"] is not None:
            x = (x + s["r"].double()).to(s["x"].dtype).double()
        root = torch.sqrt(x.pow(2).sum(1, keepdim=True) / x.shape[1] + EPS)
        if case["op"] == "norm":
            y = x / root * w
            y = _fp8_64(y) if case["form"] == "fp8" else y
            return (y, x) if s["r"] is not None else (y,)
        dy = s["dy"].double()
        inner = (dy * w * x).sum(1, keepdim=True)
        dx = dy * w / root - x * inner / (x.shape[1] * root ** 3)
        return dx if s["ds"] is None else dx + s["ds"].double(), (dy * x / root).sum(0)
    if case["op"] == "matmul":
        return _fp8_64(s["x"]) @ _weights64(s["codes"], s["scales"], case["n"], case["k"]).t()
    if case["op"] == "wgrad":
        return _fp8_64(s["dy"].t()) @ _fp8_64(s["x"].t()).t()
    norm = math.sqrt(math.fsum(float(g.double().pow(2).sum()) for g in s["grads"]))
    c = min(1.0, case["max_norm"] / norm)
    return torch.tensor(norm, dtype=torch.float64, device="cuda"), torch.cat([g.double() * c for g in s["grads"]])
