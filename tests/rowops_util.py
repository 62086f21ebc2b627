"""Helpers of the row operators' GPU tests: matrices with chosen strides and
alignment, and the error bounds."""
from __future__ import annotations

import numpy as np

import oracle
from gpu_util import torch_mod

# Half a step of rounding to nearest: relative, and half the smallest value (of a
# magnitude below the normal range).
HALF = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp16": 2.0 ** -25, "bf16": 2.0 ** -134}
F32 = 2.0 ** -24
GUARD = 0x1234           # what lies around a matrix and must stay


def torch_dtype(dtype):
    torch = torch_mod()
    return {"fp16": torch.float16, "bf16": torch.bfloat16}[dtype]


class Mat:
    """A [M, N] view of 16-bit values, rows `ld` apart, its first `shift` elements
    into the allocation; everything around it holds a guard pattern."""

    def __init__(self, M, N, dtype, ld=None, shift=0, values=None):
        torch = torch_mod()
        self.M, self.N, self.dtype = M, N, dtype
        self.ld = N if ld is None else ld
        self.shift = shift
        n = shift + max(M - 1, 0) * self.ld + N + 16
        self.raw = torch.full((n,), GUARD, dtype=torch.int16, device="cuda")
        self.t = self.raw.view(torch_dtype(dtype)).as_strided((M, N), (self.ld, 1), shift)
        if values is not None:
            self.t.copy_(values)

    def bits(self):
        torch = torch_mod()
        return self.raw.as_strided((self.M, self.N), (self.ld, 1), self.shift).cpu().numpy().view(np.uint16).copy() \
            if self.M and self.N else np.zeros((self.M, self.N), np.uint16)

    def values(self):
        return oracle.decode(self.bits(), self.dtype).astype(np.float64)

    def guards_stand(self, rows=None):
        """Whether everything outside the matrix (or outside the given rows of it) is as it was."""
        inside = np.zeros(self.raw.numel(), bool)
        for i in range(self.M) if rows is None else rows:
            at = self.shift + i * self.ld
            inside[at:at + self.N] = True
        raw = self.raw.cpu().numpy()
        return bool((raw[~inside] == GUARD).all())


# The smallest magnitude that rounds to infinity: half a step above the largest value.
OVERFLOW = {"fp16": 65520.0, "bf16": 2.0 ** 128 * (1 - 2.0 ** -9)}


def close(got, want, bound, what, dtype=None):
    """|got - want| <= bound. A result in 16 bits (dtype) is infinite where a value that near to
    `want` rounds to infinity, that is from |want| + bound >= OVERFLOW on."""
    got, want, bound = np.broadcast_arrays(np.asarray(got, np.float64), want, bound)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=what)
    ok = np.isnan(want)
    with np.errstate(invalid="ignore"):
        ok = ok | (np.abs(got - want) <= bound)
        if dtype is not None:
            ok = ok | (np.isinf(got) & (np.sign(got) == np.sign(want)) & (np.abs(want) + bound >= OVERFLOW[dtype]))
    if not ok.all():
        i = np.unravel_index(int(np.argmax(np.where(ok, 0, np.abs(got - want) / np.maximum(bound, 1e-300)))), got.shape)
        raise AssertionError(f"{what}: {int((~ok).sum())} of {got.size} outside the bound; at {i}: {got[i]!r}, "
                             f"want {want[i]!r} within {bound[i]!r}")


def rounded(want, dtype, extra):
    """Bound of a result rounded once to dtype after an error of `extra`."""
    return HALF[dtype] * (np.abs(want) + extra) + TINY[dtype] + extra
