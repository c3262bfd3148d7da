"""8-bit floating point in blocks of 128 and the gated unit, in numpy and 64 bits.

Written from the formats' definitions (sign, 4 or 5 exponent bits, 3 or 2 fraction
bits, bias 7 or 15; e4m3 has no infinity and one NaN code a sign) and the formulas,
with a table of all 256 codes in place of bit tricks.
"""
from __future__ import annotations

import numpy as np

E4M3, E5M2 = 0, 1
POW2, F32 = 0, 1
BLOCK = 128
MOST = {E4M3: 448.0, E5M2: 57344.0}


def table(fmt):
    """The value of every code, 0 to 255."""
    fraction, bias = (3, 7) if fmt == E4M3 else (2, 15)
    out = np.empty(256)
    for code in range(256):
        sign = -1.0 if code & 0x80 else 1.0
        f = code & ((1 << fraction) - 1)
        e = (code & 0x7F) >> fraction
        if fmt == E4M3 and code & 0x7F == 0x7F:
            v = np.nan
        elif fmt == E5M2 and e == 31:
            v = np.nan if f else np.inf
        elif e == 0:
            v = f * 2.0 ** (1 - bias - fraction)
        else:
            v = (1 + f / (1 << fraction)) * 2.0 ** (e - bias)
        out[code] = sign * v
    return out


def decode(q, fmt):
    return table(fmt)[np.asarray(q, np.uint8)]


def finite_codes(fmt):
    """Values of the non-negative finite codes, ascending: codes 0, 1, 2, ..."""
    t = table(fmt)[:128]
    return t[: int(np.sum(np.isfinite(t)))]


def encode(v, fmt):
    """Nearest code, ties to the even one; beyond the largest value the largest."""
    v = np.asarray(v, np.float64)
    vals = finite_codes(fmt)
    a = np.minimum(np.abs(v), vals[-1])
    hi = np.clip(np.searchsorted(vals, np.nan_to_num(a)), 1, len(vals) - 1)
    lo = hi - 1
    down, up = a - vals[lo], vals[hi] - a
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = code | np.where(np.signbit(v), 0x80, 0)
    return np.where(np.isnan(v), 0x7F, code).astype(np.uint8)


def step_at(v, fmt):
    """The distance of the format's values around v."""
    vals = finite_codes(fmt)
    i = np.clip(np.searchsorted(vals, np.abs(v)), 1, len(vals) - 1)
    return vals[i] - vals[i - 1]


def block_amax(x, block_rows=1):
    """The largest finite magnitude of every block."""
    x = np.where(np.isfinite(x), np.abs(np.asarray(x, np.float64)), 0.0)
    rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // BLOCK)
    full = np.zeros((nr * block_rows, nc * BLOCK))
    full[:rows, :cols] = x
    return full.reshape(nr, block_rows, nc, BLOCK).max(axis=(1, 3))


def scale_of(amax, fmt, kind):
    """The scales (values) of blocks with these largest magnitudes."""
    s = np.maximum(amax / MOST[fmt], 2.0 ** -126)
    if kind == F32:
        return s.astype(np.float32).astype(np.float64)
    e = np.ceil(np.log2(s))
    e = np.where(np.ldexp(1.0, (e - 1).astype(int)) >= s, e - 1, e)   # log2 may round up
    e = np.where(np.ldexp(1.0, e.astype(int)) < s, e + 1, e)          # or down
    return np.ldexp(1.0, e.astype(int))


def spread(s, rows, cols, block_rows=1):
    """A block's scale at each of its elements."""
    return np.repeat(np.repeat(s, block_rows, 0)[:rows], BLOCK, 1)[:, :cols]


def quantize(x, fmt, kind, block_rows=1):
    """(x / scale before rounding, scales, scales at each element) of a matrix."""
    s = scale_of(block_amax(x, block_rows), fmt, kind)
    by = spread(s, *x.shape, block_rows)
    with np.errstate(invalid="ignore"):
        return np.asarray(x, np.float64) / by, s, by


def sigmoid(g):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-g))


def swiglu(g, u):
    return g * sigmoid(g) * u


def swiglu_grad(g, u, dh):
    """(gradient of g, gradient of u)."""
    s = sigmoid(g)
    return dh * u * s * (1.0 + g * (1.0 - s)), dh * g * s
