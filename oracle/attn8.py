"""Rotary positions, the paged 8-bit cache and attention over it, in numpy and 64 bits.

Written from the definitions, token by token and head by head, with the formats' tables
of ``oracle.q8``.
"""
from __future__ import annotations

import numpy as np

from . import q8


def rotary(x, pos, freqs, pairs=False, scale=1.0, inverse=False):
    """x [tokens, heads, dim] with pair i of its first 2 len(freqs) values turned by pos * freqs[i]."""
    n = len(freqs)
    y = np.array(x, np.float64)
    angle = np.asarray(pos, np.float64)[:, None] * np.asarray(freqs, np.float64)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1.0 if inverse else 1.0)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if pairs else (slice(0, n), slice(n, 2 * n))
    u, v = x[..., a], x[..., b]
    y[..., a] = scale * (u * c - v * s)
    y[..., b] = scale * (u * s + v * c)
    return y


def places(starts, lengths, table, page, pages, tokens):
    """Of each token: None if it is no sequence's, else (sequence, position, page or None, offset)."""
    out = [None] * tokens
    for b, n in enumerate(lengths):
        for t in range(starts[b], starts[b + 1]):
            pos = int(n) - int(starts[b + 1]) + t
            out[t] = (b, pos, *place(table[b], pos, page, pages))
    return out


def place(row, pos, page, pages):
    if pos < 0 or pos >= len(row) * page or not 0 <= row[pos // page] < pages:
        return None, 0
    return int(row[pos // page]), pos % page


def row_scale(x, fmt, kind):
    """The scale of each row (last axis) of finite magnitudes' largest."""
    amax = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    return q8.scale_of(amax, fmt, kind)


def attend(q, k, v, sees, scale):
    """(out [dim], log of the sum, sum of p |v|, p) of one row: q [dim], k, v [n, dim], sees [n]."""
    k, v = k[sees], v[sees]
    if len(k) == 0:
        return np.zeros(v.shape[1]), -np.inf, np.zeros(v.shape[1]), np.zeros(0)
    s = (k @ q) * scale
    top = s.max()
    e = np.exp(s - top)
    p = e / e.sum()
    with np.errstate(invalid="ignore"):
        return p @ v, top + np.log(e.sum()), p @ np.abs(v), p
