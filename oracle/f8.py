"""Checker of the 8-bit operators, in 64 bits: the block format, the norm, rotary positions.

Test infrastructure only; written from the definitions (blocks of 128 values, the smallest power-of-two scale that brings the
largest magnitude to 448 or below, E4M3 values rounded to the nearest with ties to the even mantissa) and sharing no code with the
library.
"""
from fractions import Fraction

import numpy as np

BLOCK = 128
# magnitudes of E4M3 codes 0 .. 126 (127 is NaN): subnormals of 2^-9, then 1.mmm * 2^(e - 7)
GRID = np.array([c * 2.0 ** -9 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 10) for c in range(127)])


def _round_to_grid(a):
    """Code of the nearest grid value; of two equally near ones the even code (its last mantissa bit is 0)."""
    lo = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 126)
    hi = np.minimum(lo + 1, 126)
    dl, dh = a - GRID[lo], GRID[hi] - a
    return np.where((dh < dl) | ((dh == dl) & (lo % 2 == 1)), hi, lo)


def quantize(x):
    """[rows, K] -> (codes [rows, blocks, 128] 0..255, scale exponents [rows, blocks] 0..255)."""
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
    for at in zip(*np.nonzero(top)):
        n = -127
        while top[at] > 448.0 * 2.0 ** n:
            n += 1
        e[at] = n
    z = y / np.exp2(e.astype(np.float64))[..., None]
    codes = _round_to_grid(np.abs(z)) | (np.signbit(z).astype(int) << 7)
    codes[bad] = 0
    return codes.astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, exps, k=None):
    """What codes and exponents stand for, [rows, K] float64."""
    v = GRID[np.minimum(codes & 127, 126)] * np.where(codes & 128, -1.0, 1.0)
    s = np.where(exps == 255, np.nan, np.exp2(exps.astype(np.float64) - 127))
    v = (v * s[..., None]).reshape(codes.shape[0], -1)
    return v if k is None else v[:, :k]


def rounded(x):
    """x [..., K] rounded to the format, float64."""
    x = np.asarray(x, dtype=np.float64)
    flat = x.reshape(-1, x.shape[-1])
    return values(*quantize(flat), x.shape[-1]).reshape(x.shape)


def scale_at(rows, blocks):
    """Byte of the scale tiles for every (row, block)."""
    r, b = np.arange(rows)[:, None], np.arange(blocks)[None, :]
    kt = -(-blocks // 4)
    return ((r // 128) * kt + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4


def norm_rms(x, residual, weight, eps):
    """(x + residual, its norm), [rows, K]."""
    h = np.asarray(x, dtype=np.float64) + (0.0 if residual is None else np.asarray(residual, dtype=np.float64))
    y = h / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    return h, y if weight is None else y * np.asarray(weight, dtype=np.float64)


def turns(position, step):
    """Fraction of a turn in [-1/2, 1/2) of an integer position and a step of 2^64 times the turns per position, exactly."""
    n = (int(position) * int(step)) % 2 ** 64
    return float(Fraction(n - 2 ** 64 if n >= 2 ** 63 else n, 2 ** 64))


def rotate(x, positions, steps, axis, adjacent, back=False):
    """x [B, T, heads, D], positions [axes, B, T]."""
    x = np.asarray(x, dtype=np.float64)
    p = len(steps)
    angle = np.array([[[2 * np.pi * turns(positions[a, b, t], s) for s, a in zip(steps, axis)] for t in range(x.shape[1])]
                      for b in range(x.shape[0])])[:, :, None]
    c, s = np.cos(angle), np.sin(angle) * (-1 if back else 1)
    first, second = (slice(0, 2 * p, 2), slice(1, 2 * p, 2)) if adjacent else (slice(0, p), slice(p, 2 * p))
    out = x.copy()
    u, v = x[..., first], x[..., second]
    out[..., first], out[..., second] = u * c - v * s, u * s + v * c
    return out
