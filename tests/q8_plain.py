"""Plain implementations of the 8-bit operators and the rotation (numpy on the CPU): codes by fp32 operations rounded one by
one, everything else in 64 bits."""
import numpy as np

PER_CODE = np.float32(1.0) / np.float32(127.0)
TINY = np.float32(2.0 ** -126)


def codes(x):
    """x: numbers of one unit, any shape -> (codes as float64, scale as float32)."""
    x = np.asarray(x, dtype=np.float32)
    top = np.abs(x).max() if x.size else np.float32(0)
    if not np.isfinite(x).all():
        return np.zeros(x.shape), np.float32(np.nan)
    s = max(np.float32(top * PER_CODE), TINY)
    r = np.float32(1.0) / s
    return np.rint((x * r).astype(np.float32)).astype(np.float64), s


def code_rows(x):
    """codes() of every row of a matrix, at once."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        fine = np.isfinite(x).all(1)
        s = np.maximum((np.abs(x).max(1) * PER_CODE).astype(np.float32), TINY)
        y = np.rint((x * (np.float32(1.0) / s)[:, None]).astype(np.float32)).astype(np.float64)
    y[~fine], s[~fine] = 0, np.nan
    return y, s.astype(np.float32)


def prefix_quantize(x, begin, end, block, old_codes, old_scale):
    """x [B, P, Hkv, Dh] -> codes [B, P, Hkv, Dh], scale [B, Hkv, blocks]."""
    c, s = old_codes.astype(np.float64).copy(), old_scale.copy()
    B, P, Hkv, _ = x.shape
    for b in range(B):
        lo, hi = min(max(begin[b], 0), P), min(max(end[b], 0), P)
        for j in range(lo // block, -(-hi // block)) if lo < hi else ():
            t = slice(j * block, min(hi, (j + 1) * block))
            for h in range(Hkv):
                c[b, t, h], s[b, h, j] = codes(x[b, t, h])
    return c, s


def rotate(x, position, frequency, weight, eps, interleaved, gain):
    """x [T, H, Dh] float64 -> norm and rotation in 64 bits, and the size of each result's terms (for error bounds)."""
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    y, size = x.copy(), np.abs(x)
    half = len(frequency)
    u = np.asarray(position, dtype=np.float64)[:, None] * frequency
    c, s = (gain * np.cos(u))[:, None], (gain * np.sin(u))[:, None]
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = gain * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, size


def head(hidden, w_codes, w_scale):
    """hidden [R, H], w_codes [V, H], w_scale [V] -> token, confidence, lse, logits (fp32 numbers)."""
    x, s = code_rows(hidden)
    n = x @ w_codes.astype(np.float64).T
    with np.errstate(invalid="ignore"):
        l = ((n.astype(np.float32) * w_scale.astype(np.float32)).astype(np.float32) * s[:, None]).astype(np.float32)
        z = l.astype(np.float64)
        m = z.max(1)
        lse = m + np.log(np.exp(z - m[:, None]).sum(1))
    return l.argmax(1), np.exp(m - lse), lse, l
