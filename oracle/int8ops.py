"""Plain 64-bit reference of the 8-bit operators: rows in 8-bit integers, the RMS norm of
a sum with its gradients, products of 8-bit matrices, alone and by experts. Written from
the formulas in include/fo.h; values in and out are float64 arrays, codes int8."""
from __future__ import annotations

import numpy as np


def quantize(x):
    """(codes [M, N], scales [M]) of x [M, N]: 127 x / m to nearest even, m / 127. (127 x is
    exact in 64 bits, and a quotient of such numbers that is no tie is not rounded to one.)"""
    finite = np.isfinite(x).all(axis=1)
    v = np.where(finite[:, None], x, 0.0)
    m = np.abs(v).max(axis=1, initial=0.0)
    codes = np.rint(127.0 * v / np.where(m > 0, m, 1.0)[:, None])
    return codes.astype(np.int8), np.where(finite, m / 127.0, np.nan)


def norm_add(h, gamma, eps):
    """(rstd [M], y [M, N]) of h as it is kept."""
    rstd = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
    return rstd, h * rstd[:, None] * (1.0 if gamma is None else gamma)


def norm_add_grad(dy, dh, h, gamma, rstd):
    """(dx, dgamma), rstd taken as a function of h with the given values."""
    g = dy if gamma is None else dy * gamma
    hat = h * rstd[:, None]
    dx = rstd[:, None] * (g - hat * (g * hat).mean(axis=1, keepdims=True))
    return dx if dh is None else dh + dx, (dy * hat).sum(axis=0)


def product(a, a_scales, b, b_scales, bias=None):
    """(c, magnitude of the product) of codes a [M, K], b [N, K]."""
    sums = a.astype(np.float64) @ b.astype(np.float64).T
    c = sums * a_scales.astype(np.float64)[:, None] * b_scales.astype(np.float64)
    return (c if bias is None else c + bias), np.abs(c)


def experts(a, a_scales, b, b_scales, offsets, counts, capacity, pair_of=None, choices=1, bias=None):
    """{row: (values, magnitude)} of the rows that are written: b [E, N, K]."""
    out, pair_of = {}, None if pair_of is None else np.asarray(pair_of)
    for e in range(len(counts)):
        rows = np.arange(int(offsets[e]), min(int(offsets[e]) + int(counts[e]), capacity))
        src = rows if pair_of is None else np.where(pair_of[rows] >= 0, pair_of[rows] // choices, -1)
        rows, src = rows[(src >= 0) & (src < len(a))], src[(src >= 0) & (src < len(a))]
        if len(rows):
            c, mag = product(a[src], a_scales[src], b[e], b_scales[e], None if bias is None else bias[e])
            out.update((int(r), (c[i], mag[i])) for i, r in enumerate(rows))
    return out
