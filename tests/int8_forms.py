"""Which kernel and blocks a product of 8-bit matrices takes, from the header that the
library is built from; and the sizes at which the tests reach every one of them."""
from __future__ import annotations

import ctypes
import os
import subprocess

import paper_2504_19519_amd as fo

CSRC = os.path.join(os.path.dirname(os.path.abspath(fo.__file__)), "csrc")
INCLUDE = os.path.join(os.path.dirname(os.path.dirname(CSRC)), "include")

HARNESS = r"""
#include "int8_form.h"
static void put(const fo::Int8Args& a, const fo::Int8Form& f, bool experts, int32_t* out) {
    out[0] = f.rows; out[1] = f.cols; out[2] = f.stages; out[3] = f.parts; out[4] = f.span;
    out[5] = f.cols <= 64 && f.rows > 16 && fo::weights_once(a, f, experts);
}
extern "C" void product(int64_t M, int64_t N, int64_t K, int64_t ldb, int32_t* out) {
    fo::Int8Args a{};
    a.M = M; a.N = N; a.K = K; a.ldb = ldb;
    put(a, fo::product_form(M, N, K), false, out);
}
extern "C" void experts(int64_t capacity, int64_t N, int64_t K, int64_t ldb, int32_t E, int64_t a_rows, int32_t choices, int gather,
                        int32_t* out) {
    fo::Int8Args a{};
    a.M = capacity; a.N = N; a.K = K; a.ldb = ldb; a.E = E; a.a_rows = a_rows; a.choices = choices; a.capacity = (int32_t)capacity;
    a.pair_of = gather ? out : nullptr;
    put(a, fo::experts_form(a), true, out);
}
"""


def row_bytes(n):
    return -(-n // 16) * 16


class Rules:
    """The rules, built by the host's compiler in directory `d`."""

    def __init__(self, d):
        src, lib = os.path.join(d, "forms.cpp"), os.path.join(d, "forms.so")
        with open(src, "w") as f:
            f.write(HARNESS)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, "-I", INCLUDE, src, "-o", lib], check=True)
        self.lib = ctypes.CDLL(lib)
        i64, i32 = ctypes.c_int64, ctypes.c_int32
        self.lib.product.argtypes = [i64] * 4 + [ctypes.c_void_p]
        self.lib.experts.argtypes = [i64] * 4 + [i32, i64, i32, ctypes.c_int, ctypes.c_void_p]

    @staticmethod
    def name(out, experts):
        rows, cols, stages, parts, span, once = out
        text = {16: "few", 256: "tile"}.get(rows, f"{rows}x{cols}/{stages}")
        return text + (f" parts {parts}" if parts > 1 else "") + (f" span {span}" if experts and rows < 256 else "") + (" once" if once else "")

    def product(self, M, N, K, ldb=None):
        out = (ctypes.c_int32 * 6)()
        self.lib.product(M, N, K, row_bytes(K) if ldb is None else ldb, out)
        return self.name(out, False)

    def experts(self, capacity, N, K, E, rows, choices, gather, ldb=None):
        out = (ctypes.c_int32 * 6)()
        self.lib.experts(capacity, N, K, row_bytes(K) if ldb is None else ldb, E, rows, choices, gather, out)
        return self.name(out, True)


# Products: the form, M, N, K, and the distance of b's rows where it is not K rounded up to 16.
PRODUCTS = [
    ("few", 1, 1000, 515, None), ("few", 16, 256, 1024, None), ("few", 3, 4090, 9001, None),
    ("32x32/4", 30, 9001, 300, None), ("32x32/4", 7, 5000, 129, None),
    ("32x32/4 parts 4", 31, 515, 8300, None), ("32x32/4 parts 4", 128, 1000, 8177, None),
    ("32x32/4 once", 30, 16500, 8192, None),
    ("32x32/4 parts 4 once", 20, 4000, 34000, 34048),
    ("64x32/4", 128, 4096, 1024, None), ("64x32/4", 100, 3001, 1000, None),
    ("64x32/4 once", 60, 8000, 17000, 17024),
    ("64x64/4", 120, 6000, 260, None), ("64x64/4", 33, 9000, 500, None),
    ("64x64/4 once", 59, 9201, 15809, 15872),
    ("128x64/3", 333, 3000, 700, None), ("128x64/3", 129, 8200, 40, None),
    ("128x64/3 once", 75, 10751, 12506, 12544),
    ("128x128/3", 1024, 4096, 1024, None), ("128x128/3", 1000, 4090, 1300, None), ("128x128/3", 669, 3087, 949, None),
    ("128x128/2", 2048, 2304, 512, None), ("128x128/2", 4000, 4090, 700, None),
    # one, two, three and more tiles to a workgroup, whole and with ends of rows, columns and sums
    ("tile", 4096, 4096, 2048, None), ("tile", 1587, 5533, 1471, None), ("tile", 6511, 2568, 1442, None), ("tile", 4096, 8192, 1024, None),
    ("tile", 10426, 3153, 566, 640), ("tile", 5258, 9392, 292, None), ("tile", 7677, 15863, 100, None),
]

# Experts: the form, T tokens to K of E experts, N columns, H inner values, whether rows are taken through
# the pairs, the padding, and the distance of b's rows.
EXPERTS = [
    ("32x32/4 span 1", 40, 4, 60, 70, 200, True, 1, None), ("32x32/4 span 1", 500, 4, 200, 64, 70, False, 1, None),
    ("32x32/4 span 1 once", 11, 3, 8, 3470, 4741, True, 1, 4864), ("32x32/4 span 1 once", 6, 3, 16, 781, 10673, False, 1, 10752),
    ("64x64/4 span 1", 2100, 4, 256, 64, 300, True, 1, None), ("64x64/4 span 1", 16, 8, 256, 600, 300, False, 1, None),
    ("64x64/4 span 1 once", 16, 8, 256, 1100, 1024, True, 1, None), ("64x64/4 span 1 once", 48, 3, 128, 2931, 261, False, 1, 384),
    ("64x64/4 span 4", 200, 4, 160, 2530, 300, True, 1, None), ("64x64/4 span 4", 200, 4, 160, 2499, 900, False, 1, None),
    ("64x64/4 span 4 once", 193, 2, 200, 5261, 100, True, 1, 128), ("64x64/4 span 4 once", 307, 1, 256, 4360, 120, False, 1, 128),
    ("128x128/2 span 1", 700, 4, 8, 2300, 300, True, 1, None), ("128x128/2 span 1", 1217, 4, 20, 1100, 1409, False, 64, None),
    ("128x128/2 span 2", 2165, 1, 256, 931, 266, True, 1, None), ("128x128/2 span 2", 718, 4, 256, 900, 320, False, 1, None),
    ("128x128/2 span 4", 160, 4, 60, 4467, 13, True, 1, None), ("128x128/2 span 4", 150, 4, 60, 4545, 9, False, 1, None),
    ("tile", 3000, 2, 3, 2990, 600, True, 1, None), ("tile", 1706, 2, 2, 5363, 785, True, 16, None), ("tile", 2087, 1, 1, 6065, 2055, False, 1, None),
    ("tile", 4096, 2, 8, 4608, 512, False, 64, None), ("tile", 4096, 2, 8, 2048, 1100, True, 1, None),
]


def expert_rows(T, K, E, align):
    """fo_route_capacity."""
    return T * K + min(E, T * K) * (align - 1)


# The longest sums, K = 131071, undivided but for the one in parts: the form, M, N.
LONGEST = [("few", 4, 2100), ("32x32/4 once", 20, 4200), ("32x32/4 parts 4", 40, 20), ("64x32/4 once", 60, 4200), ("64x64/4 once", 40, 8300),
           ("128x64/3 once", 100, 8300), ("128x128/3", 1500, 1600), ("128x128/2", 2100, 2100), ("tile", 2560, 4000)]
# by experts: the form, rows of each, N
LONGEST_EXPERTS = [("32x32/4 span 1", (5, 0, 3), 200), ("32x32/4 span 1 once", (20, 30, 1), 700), ("128x128/2 span 1", (700, 0, 800), 1500), ("tile", (2500, 60), 3300),
                   ("64x64/4 span 1 once", (1,) * 40, 1700)]

# A block whose projection and experts' products all go in tiles of 256 x 256, more than the 256 compute units:
# T tokens to K of E experts, H values, F inner ones, Q columns of the projection.
TILED_BLOCK = dict(T=4096, K=2, E=4, H=2000, F=2304, Q=4400)
