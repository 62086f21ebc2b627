"""Plain 64-bit reference of the row operators: norms and their gradients, 8-bit
checkpoints, tokens sorted by expert and combined. Written from the formulas in
include/fo.h; values in and out are float64 arrays (codes and scales uint8)."""
from __future__ import annotations

import numpy as np

BLOCK = 32
EMAX = {"fp16": 15, "bf16": 127}


def norm_stats(x, kind, eps):
    """(mean, rstd) of the rows of x [M, N]."""
    mean = x.mean(axis=1) if kind == "layer" else np.zeros(len(x))
    return mean, 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)


def norm(x, mean, rstd, gamma, beta):
    y = (x - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * gamma
    return y if beta is None else y + beta


def norm_grad(dy, x, mean, rstd, gamma, kind):
    """(dx, dgamma, dbeta), the statistics taken as functions of x with the given values."""
    h = (x - mean[:, None]) * rstd[:, None]
    g = dy if gamma is None else dy * gamma
    dx = g - h * (g * h).mean(axis=1, keepdims=True)
    if kind == "layer":
        dx = dx - g.mean(axis=1, keepdims=True)
    return dx * rstd[:, None], (dy * h).sum(axis=0), dy.sum(axis=0)


def _to_e4m3(z):
    """Codes of values with |z| <= 448, to nearest even: 4 exponent bits (bias 7), 3 of the fraction."""
    a = np.abs(z)
    _, e = np.frexp(a)
    step_exp = np.maximum(e - 4, -9)
    n = np.rint(np.ldexp(a, -step_exp)).astype(np.int64)      # value = n * 2^step_exp, n <= 16
    up = n == 16
    n, step_exp = np.where(up, 8, n), np.where(up, step_exp + 1, step_exp)
    field = np.where(n >= 8, step_exp + 10, 0)                # 1.xxx * 2^(field - 7) = n * 2^(field - 10)
    code = (field << 3) | (n & 7)
    return (code | (np.signbit(z).astype(np.int64) << 7)).astype(np.uint8)


def _from_e4m3(code):
    c = code.astype(np.int64)
    field, n = (c >> 3) & 15, c & 7
    value = np.where(field > 0, np.ldexp(8.0 + n, field - 10), np.ldexp(1.0 * n, -9))
    return np.where(c & 128, -value, value)


def pack(x, fmt, dtype):
    """(codes [M, B * 32], scales [M, B]) of x [M, N], whose values are dtype's."""
    M, N = x.shape
    B = -(-N // BLOCK)
    v = np.zeros((M, B * BLOCK))
    v[:, :N] = x
    v = v.reshape(M, B, BLOCK)
    finite = np.isfinite(v).all(axis=2)
    v = np.where(finite[:, :, None], v, 0.0)
    top = np.abs(v).max(axis=2)
    m, e = np.frexp(top)                                      # top = m * 2^e, m in [1/2, 1)
    e = np.where(top > 0, e - 1, -1000)
    if fmt == "int8":
        s = np.maximum(e - 6, -126)
        codes = np.clip(np.rint(np.ldexp(v, -s[:, :, None])), -127, 127).astype(np.int8).view(np.uint8)
    else:
        up = 2.0 * m > 1.75
        s = np.maximum(e - 8 + up, -126)
        limit = np.where(up & (e == EMAX[dtype]), 240.0, 448.0)[:, :, None]
        codes = _to_e4m3(np.clip(np.ldexp(v, -s[:, :, None]), -limit, limit))
    return codes.reshape(M, B * BLOCK), np.where(finite, s + 127, 255).astype(np.uint8)


def unpack(codes, scales, N, fmt):
    """What a checkpoint stands for, [M, N]."""
    M, B = scales.shape
    c = codes.reshape(M, B, BLOCK)
    v = c.view(np.int8).astype(np.float64) if fmt == "int8" else _from_e4m3(c)
    v = np.ldexp(v, scales.astype(np.int64)[:, :, None] - 127)
    return np.where(scales[:, :, None] == 255, np.nan, v).reshape(M, B * BLOCK)[:, :N]


def route_sort(ids, E, align):
    """(offsets, counts, slot_of, pair_of up to offsets[E]) of ids [T, K]."""
    flat = ids.reshape(-1)
    counts = np.array([(flat == e).sum() for e in range(E)], np.int64)
    offsets = np.concatenate([[0], np.cumsum(-(-counts // align) * align)]).astype(np.int64)
    slot, pair = np.full(flat.shape, -1, np.int64), np.full(int(offsets[E]), -1, np.int64)
    nxt = offsets[:E].copy()
    for p, e in enumerate(flat):
        if 0 <= e < E:
            slot[p] = nxt[e]
            pair[nxt[e]] = p
            nxt[e] += 1
    return offsets, counts, slot.reshape(ids.shape), pair


def combine(rows, slot, w):
    """(out, sum of magnitudes): pairs with a row only."""
    T, K = slot.shape
    out, mag = np.zeros((T, rows.shape[1])), np.zeros((T, rows.shape[1]))
    for t in range(T):
        for k in range(K):
            if 0 <= slot[t, k] < len(rows):
                v = rows[slot[t, k]] * (1.0 if w is None else w[t, k])
                out[t] += v
                mag[t] += np.abs(v)
    return out, mag


def combine_grad(dout, rows, slot, w, capacity):
    """({row: its gradient}, dweights, sums of magnitudes of dweights)."""
    T, K = slot.shape
    drows, dw, mag = {}, np.zeros((T, K)), np.zeros((T, K))
    for t in range(T):
        for k in range(K):
            s = int(slot[t, k])
            if 0 <= s < capacity:
                drows[s] = dout[t] * (1.0 if w is None else w[t, k])
                if rows is not None:
                    dw[t, k] = (dout[t] * rows[s]).sum()
                    mag[t, k] = np.abs(dout[t] * rows[s]).sum()
    return drows, dw, mag
