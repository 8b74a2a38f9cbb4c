"""The learner-side operators in 64 bits, element by element from their definitions (numpy; test code)."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GELU_A, GELU_B = np.sqrt(2.0 / np.pi), 0.044715


def block_scales(x, below):
    """Scale byte of every block of 32 along the rows of a float32 matrix."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    nb = -(-cols // 32)
    s = np.zeros((rows, nb), dtype=np.int64)
    for b in range(nb):
        part = np.abs(x[:, 32 * b:32 * b + 32].astype(np.float64))
        bad = ~np.isfinite(part).all(axis=1)
        top = np.where(np.isfinite(part), part, 0.0).max(axis=1)
        exponent = np.frexp(top)[1] - 1                       # floor(log2 top)
        s[:, b] = np.where(top > 0, np.maximum(exponent + 127 - below, 0), 0)
        s[bad, b] = 255
    return s


def _scaled(x, s):
    x = np.asarray(x, dtype=np.float32).astype(np.float64)
    per = np.repeat(s, 32, axis=1)[:, :x.shape[1]]
    return np.where(per == 255, 0.0, np.where(np.isfinite(x), x, 0.0) * np.exp2(127.0 - per)), per


def values(codes, s):
    per = np.repeat(s, 32, axis=1)[:, :codes.shape[1]]
    return np.where(per == 255, np.nan, codes * np.exp2(np.minimum(per, 254) - 127.0))


def mx4(x):
    """(signed E2M1 magnitudes with their signs, indices 0..15 of the codes, scale bytes)."""
    s = block_scales(x, 2)
    v, _ = _scaled(x, s)
    a = np.minimum(np.abs(v), 6.0)
    d = np.abs(a[..., None] - GRID)
    near = d.min(axis=-1, keepdims=True)
    tied = d == near
    even = tied & (np.arange(8) % 2 == 0)
    index = np.where(even.any(axis=-1), even.argmax(axis=-1), tied.argmax(axis=-1))
    negative = np.signbit(np.where(np.isnan(x), 0.0, np.asarray(x, dtype=np.float32))) & (np.repeat(s, 32, axis=1)[:, :v.shape[1]] != 255)
    return np.where(negative, -1.0, 1.0) * GRID[index], index + 8 * negative, s


def mx4_bytes(x):
    """(codes, scales) as the library lays them out; padding scale rows are zero here."""
    rows, cols = x.shape
    _, index, s = mx4(x)
    nb = s.shape[1]
    full = np.zeros((rows, nb * 32), dtype=np.uint8)
    full[:, :cols] = index
    codes = full[:, 0::2] | (full[:, 1::2] << 4)
    kt = -(-nb // 4)
    scales = np.zeros(-(-rows // 128) * kt * 512, dtype=np.uint8)
    r, b = np.meshgrid(np.arange(rows), np.arange(nb), indexing="ij")
    scales[mx4_scale_at(r, b, kt)] = s
    return codes, scales


def mx4_scale_at(r, b, kt):
    return ((r // 128) * kt + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4


def mx4_values(x):
    v, _, s = mx4(x)
    return values(v, s)


def act8(x):
    s = block_scales(x, 6)
    v, _ = _scaled(x, s)
    return np.clip(np.rint(v), -127, 127), s


def act8_values(x):
    c, s = act8(x)
    return values(c, s)


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def sigmoid_argument(act, x):
    return 2.0 * GELU_A * (x + GELU_B * x ** 3) if act == "gelu" else x


def f(act, x):
    if act == "relu":
        return np.maximum(x, 0.0)
    return x * sigmoid(sigmoid_argument(act, x))


def slope(act, x):
    if act == "relu":
        return (x > 0).astype(np.float64)
    s = sigmoid(sigmoid_argument(act, x))
    du = 2.0 * GELU_A * (1.0 + 3.0 * GELU_B * x ** 2) if act == "gelu" else 1.0
    return s + x * s * (1.0 - s) * du
