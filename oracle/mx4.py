"""Checker of the 4-bit operators, in 64 bits: the block format, the product of such operands, attention over them.

Test infrastructure only; written from the definitions (blocks of 32 values, scale 2^(floor(log2 max) - 2), E2M1 values
rounded to the nearest with ties to the even mantissa) and sharing no code with the library.
"""
import numpy as np

BLOCK = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _round_to_grid(a):
    """Index of the nearest grid value; of two equally near ones the even index (its mantissa bit is 0)."""
    lo = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 7)
    hi = np.minimum(lo + 1, 7)
    dl, dh = a - GRID[lo], GRID[hi] - a
    return np.where((dh < dl) | ((dh == dl) & (lo % 2 == 1)), hi, lo)


def quantize(x):
    """[rows, K] -> (codes [rows, blocks, 32] 0..15, scale exponents [rows, blocks] 0..255)."""
    x = np.asarray(x, dtype=np.float64)
    rows, k = x.shape
    nb = -(-k // BLOCK)
    y = np.zeros((rows, nb * BLOCK))
    y[:, :k] = x
    y = y.reshape(rows, nb, BLOCK)
    bad = ~np.isfinite(y).all(-1)
    y = np.where(bad[..., None], 0.0, y)
    top = np.abs(y).max(-1)
    e = np.full(top.shape, -127)
    live = top > 0
    e[live] = np.maximum(np.floor(np.log2(top[live])).astype(int) - 2, -127)
    # (log2 of a value just below a power of two may round up to it)
    over = live & (e > -127) & (top < np.exp2(e + 2.0))
    e[over] -= 1
    z = y / np.exp2(e.astype(np.float64))[..., None]
    codes = _round_to_grid(np.abs(z)) | (np.signbit(z).astype(int) << 3)
    return codes.astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, exps, k=None):
    """What codes and exponents stand for, [rows, K] float64."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(exps == 255, np.nan, np.exp2(exps.astype(np.float64) - 127))
    v = (v * s[..., None]).reshape(codes.shape[0], -1)
    return v if k is None else v[:, :k]


def rounded(x):
    """x [..., K] rounded to the format, float64."""
    x = np.asarray(x, dtype=np.float64)
    flat = x.reshape(-1, x.shape[-1])
    return values(*quantize(flat), x.shape[-1]).reshape(x.shape)


def attend(q, k, v, group, scale, first_seen):
    """One sequence: q [T, heads, D], k and v [n, kv_heads, D]; row i sees the tokens 0 .. first_seen + i.
    Returns (result, sum of p |v| / sum p) [T, heads, D]."""
    t, heads, d = q.shape
    out, mag = np.zeros((t, heads, d)), np.zeros((t, heads, d))
    for i in range(t):
        n = min(first_seen + i + 1, k.shape[0])
        if n <= 0:
            continue
        for h in range(heads):
            s = scale * (k[:n, h // group] @ q[i, h])
            p = np.exp(s - s.max()) if np.isfinite(s).all() else np.full(n, np.nan)
            out[i, h] = p @ v[:n, h // group] / p.sum()
            mag[i, h] = p @ np.abs(v[:n, h // group]) / p.sum()
    return out, mag
