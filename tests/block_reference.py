"""FP8 in blocks of 128, the norm and the clipping in 64 bits, from their definitions (numpy; test code)."""
import numpy as np

#: the non-negative E4M3 numbers in the order of their codes
E4M3 = np.array([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)])


def scale_at(r, b, kt):
    return ((r // 128) * kt + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4


def block_scales(x, square=False):
    """Scale byte of every row and block of 128 of a float32 matrix."""
    x = np.asarray(x, dtype=np.float32).astype(np.float64)
    rows, cols = x.shape
    nb = -(-cols // 128)
    s = np.zeros((rows, nb), dtype=np.int64)
    step = 128 if square else 1
    for b in range(nb):
        for r in range(0, rows, step):
            part = np.abs(x[r:r + step, 128 * b:128 * b + 128])
            if not np.isfinite(part).all():
                s[r:r + step, b] = 255
                continue
            p = -127
            while part.max() > 448.0 * 2.0 ** p:
                p += 1
            s[r:r + step, b] = p + 127
    return s


def fp8(x, square=False):
    """(codes, scale bytes per row and block) of a float32 matrix."""
    x = np.asarray(x, dtype=np.float32)
    s = block_scales(x, square)
    per = np.repeat(s, 128, axis=1)[:, :x.shape[1]]
    a = np.abs(np.where(np.isfinite(x), x, 0.0).astype(np.float64)) * np.exp2(127.0 - per)
    low = np.clip(np.searchsorted(E4M3, a, side="right") - 1, 0, len(E4M3) - 2)
    mid = (E4M3[low] + E4M3[low + 1]) / 2
    code = low + ((a > mid) | ((a == mid) & (low % 2 == 1)))
    code = np.where(per == 255, 0, code + 128 * np.signbit(np.where(np.isnan(x), 0.0, x)))
    return code, s


def values(code, s):
    per = np.repeat(s, 128, axis=1)[:, :code.shape[1]]
    v = np.where(code >= 128, -1.0, 1.0) * E4M3[code % 128]
    return np.where(per == 255, np.nan, v * np.exp2(np.minimum(per, 254) - 127.0))


def fp8_values(x, square=False):
    return values(*fp8(x, square))


def fp8_bytes(x, square=False):
    """(codes, scales) as the library lays them out; scale bytes of rows past the last are zero here."""
    rows, cols = x.shape
    code, s = fp8(x, square)
    nb = s.shape[1]
    codes = np.zeros((rows, nb * 128), dtype=np.uint8)
    codes[:, :cols] = code
    kt = -(-nb // 4)
    scales = np.zeros(-(-rows // 128) * kt * 512, dtype=np.uint8)
    r, b = np.meshgrid(np.arange(rows), np.arange(nb), indexing="ij")
    scales[scale_at(r, b, kt)] = s
    return codes, scales


def norm(s, w, eps):
    s, w = np.asarray(s, dtype=np.float64), np.asarray(w, dtype=np.float64)
    return s * w / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps)


def norm_backward(dy, s, w, eps, dsum=None):
    """(ds, dw, and the sums of magnitudes that their errors go by)."""
    dy, s, w = (np.asarray(v, dtype=np.float64) for v in (dy, s, w))
    r = 1.0 / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps)
    ds = r * (w * dy - s * r * r * (w * dy * s).mean(axis=1, keepdims=True))
    size = r * (np.abs(w * dy) + np.abs(s) * r * r * np.abs(w * dy * s).mean(axis=1, keepdims=True))
    if dsum is not None:
        ds, size = ds + dsum, size + np.abs(dsum)
    return ds, (dy * s * r).sum(axis=0), size, np.abs(dy * s * r).sum(axis=0)


def clip(grads, max_norm):
    """(norm, what the gradients become)."""
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        n = np.sqrt(sum((np.asarray(g, dtype=np.float64) ** 2).sum() for g in grads))
        by = 1.0 if np.float32(n) <= max_norm else max_norm / n
        return n, [np.asarray(g, dtype=np.float64) * by for g in grads]
