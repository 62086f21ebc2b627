"""Helpers of the 8-bit operators' GPU tests: matrices of codes, vectors, and the checks
of each operator's outputs with their bounds."""
from __future__ import annotations

import numpy as np

import oracle
from gpu_util import torch_mod
from oracle import int8ops as ref
from rowops_util import F32, HALF, TINY, close, rounded

GUARD8 = 0x5A


def row_bytes(n):
    return -(-n // 16) * 16


class Codes:
    """A [M, N] matrix of codes, rows `ld` bytes apart, behind `shift` bytes; everything
    around its rows' whole chunks of 16 holds a guard pattern."""

    def __init__(self, M, N, ld=None, shift=0, values=None):
        torch = torch_mod()
        self.M, self.N, self.width = M, N, row_bytes(N)
        self.ld = self.width if ld is None else ld
        self.shift = shift
        n = shift + max(M - 1, 0) * self.ld + self.width + 32
        self.raw = torch.full((n,), GUARD8, dtype=torch.int8, device="cuda")
        self.whole = self.raw.as_strided((M, self.width), (self.ld, 1), shift)      # rows with what is behind their end
        self.t = self.raw.as_strided((M, N), (self.ld, 1), shift)
        if values is not None:
            self.whole.zero_()
            self.t.copy_(torch.as_tensor(values))

    def ptr(self):
        return self.raw.data_ptr() + self.shift

    def values(self):
        return self.t.cpu().numpy()

    def rest_is_zero(self):
        return not self.whole[:, self.N:].any().item()

    def guards_stand(self):
        inside = np.zeros(self.raw.numel(), bool)
        for i in range(self.M):
            inside[self.shift + i * self.ld:self.shift + i * self.ld + self.width] = True
        return bool((self.raw.cpu().numpy()[~inside] == GUARD8).all())


def f32_vec(n, value=-7.0):
    torch = torch_mod()
    return torch.full((n,), value, dtype=torch.float32, device="cuda")


def to_dtype(values, dtype):
    """float64 values rounded to 16 bits, as float64."""
    return oracle.decode(oracle.encode(np.asarray(values, np.float64), dtype), dtype).astype(np.float64)


# ---- bounds --------------------------------------------------------------------
# A sum over a row: up to 32 terms in one thread, six additions over a wave, four over
# the waves; with the products' own rounding less than 46 roundings along any path.
ROW_SUM = 46 * F32
# rstd: half of the relative error of (sum / N + eps), which has three roundings more, and the root's.
RSTD = (ROW_SUM + 3 * F32) / 2 + 1.5 * 2 * F32


def kept_sum(x, r, dtype):
    """x + residual as it is kept: in 32 bits, then in 16."""
    if r is None:
        return x
    return to_dtype((x.astype(np.float32) + r.astype(np.float32)).astype(np.float64), dtype)


def check_quantized(codes, scales, x, what):
    """Codes and scales of x: exactly those of the formula."""
    want, _ = ref.quantize(x)
    np.testing.assert_array_equal(codes, want, err_msg=what)
    # the quotient of two fp32 numbers, rounded once
    np.testing.assert_array_equal(scales, np.abs(x).max(axis=1).astype(np.float32) / np.float32(127), err_msg=what)


def check_norm_codes(codes, scales, h, gamma, rstd, what):
    """Codes of y: 127 t / max|t| with t = h gamma, which is exact in 64 bits; scale = max|t| rstd / 127."""
    t = h if gamma is None else h * gamma
    want, s = ref.quantize(t)
    np.testing.assert_array_equal(codes, want, err_msg=what)
    s = s * rstd
    close(scales, s, np.abs(s) * (RSTD + 2 * F32) + 2.0 ** -149, what)


def check_grads(dx, dgamma, dy, dh, h, gamma, rstd, dtype, what):
    want, want_gamma = ref.norm_add_grad(dy, dh, h, gamma, rstd)
    g = dy if gamma is None else dy * gamma
    M, N = h.shape
    r = rstd[:, None]
    if dx is not None:
        through = r ** 3 * np.abs(h) * np.abs(g * h).sum(axis=1, keepdims=True) / N
        extra = 4 * F32 * (np.abs(r * g) + (0.0 if dh is None else np.abs(dh))) + (ROW_SUM + 7 * F32) * through
        close(dx, want, rounded(want, dtype, extra), what + " dx", dtype)
    if dgamma is not None:
        # a thread's rows (a 64th of them at most), the row groups' and workgroups' sums, the product's three roundings
        steps = -(-M // 64) + 24 + 3
        close(dgamma, want_gamma, steps * F32 * np.abs(dy * h * r).sum(axis=0) + 2.0 ** -149, what + " dgamma")


def product_bound(want, magnitude, dtype):
    """The sum rounded to 32 bits, two products, the bias's addition; then 16 bits."""
    return rounded(want, dtype, 3 * F32 * magnitude + F32 * np.abs(want))


__all__ = [n for n in dir() if not n.startswith("_")]
