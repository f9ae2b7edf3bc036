"""Microscaled 4-bit values (MXFP4: E2M1 elements, a power of two per 32) in
float64, by search in the table of the format's values.  Test infrastructure."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def term(x):
    """x [rows][cols] -> the values of its blocks (NaN blocks whole)."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    b = np.zeros((rows, nb * BLOCK))
    b[:, :cols] = x
    b = b.reshape(rows, nb, BLOCK)
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(-1)
    exp = np.where(top > 0, np.frexp(top)[1] - 1, -1000)   # floor(log2 top)
    scale = np.ldexp(1.0, np.clip(exp - 2, -127, 127))[..., None]
    a = np.abs(b) / scale
    mids = (GRID[1:] + GRID[:-1]) / 2
    # a tie between codes i and i + 1 goes to the even one
    code = np.zeros(a.shape, dtype=np.int64)
    for i, m in enumerate(mids):
        code += (a >= m) if i % 2 else (a > m)
    v = np.copysign(GRID[code], b) * scale
    v[bad] = np.nan
    return v.reshape(rows, -1)[:, :cols]


def quantised(x, terms):
    """The values that x quantised in one or two terms stands for."""
    x = np.asarray(x, dtype=np.float64)
    hi = term(x)
    if terms == 1:
        return hi
    with np.errstate(invalid="ignore"):
        return hi + term(x - hi)


def block_same(a, b):
    """Per block of 32 columns: whether two value matrices agree in all of it."""
    rows, cols = a.shape
    nb = -(-cols // BLOCK)
    pad = np.ones((rows, nb * BLOCK), dtype=bool)
    pad[:, :cols] = (a == b) | (np.isnan(a) & np.isnan(b))
    return pad.reshape(rows, nb, BLOCK).all(-1)


def rms_norm(s, gain, eps):
    s = np.asarray(s, dtype=np.float64)
    return s / np.sqrt((s * s).mean(-1, keepdims=True) + eps) * gain


def swiglu(gate, up):
    g = np.asarray(gate, dtype=np.float64)
    e = np.exp(-np.abs(g))
    return np.where(g >= 0, g / (1 + e), g * e / (1 + e)) * np.asarray(up, dtype=np.float64)
