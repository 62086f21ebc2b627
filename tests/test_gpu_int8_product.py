"""Products of 8-bit matrices, alone and by experts, against the 64-bit reference: every
form, ragged sizes, strides, extreme codes and scales, rows that are left as they were."""
import numpy as np
import pytest

import paper_2504_19519_amd as fo
from gpu_util import torch_mod
from int8_util import Codes, product_bound, row_bytes, to_dtype
from oracle import int8ops as ref
from oracle import rowops as rowref
from rowops_util import GUARD, Mat, close, torch_dtype

pytestmark = pytest.mark.gpu
DTYPES = ["fp16", "bf16"]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = torch_mod()
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    fo.lib()
    yield
    torch.cuda.synchronize()


def dev(v):
    return torch_mod().as_tensor(np.ascontiguousarray(v)).cuda()


def vec(v, dtype):
    return None if v is None else dev(np.asarray(v)).to(torch_dtype(dtype))


def codes(rng, *shape):
    return rng.integers(-128, 128, shape).astype(np.int8)


def scales(rng, *shape):
    return np.exp2(rng.uniform(-9, -5, shape)).astype(np.float32)


def workspace(M, N, K):
    torch = torch_mod()
    return torch.full((fo.int8_workspace_bytes(M, N, K),), 0xFF, dtype=torch.uint8, device="cuda")


def run(a, sa, b, sb, bias, dtype, lda=None, ldb=None, ldc=None, shift=0):
    (M, K), N = a.shape, len(b)
    A, B, C = Codes(M, K, lda, values=a), Codes(N, K, ldb, values=b), Mat(M, N, dtype, ldc, shift)
    fo.int8_product(A.whole, dev(sa), B.whole, dev(sb), C.t, M, N, K, dtype, bias=vec(bias, dtype), workspace=workspace(M, N, K))
    assert C.guards_stand()
    return C


def check(M, N, K, dtype, seed=0, bias=False, **kw):
    rng = np.random.default_rng(seed + M + 7 * N + 13 * K)
    a, b, sa, sb = codes(rng, M, K), codes(rng, N, K), scales(rng, M), scales(rng, N)
    bv = to_dtype(rng.normal(size=N), dtype) if bias else None
    C = run(a, sa, b, sb, bv, dtype, **kw)
    want, mag = ref.product(a, sa, b, sb, bv)
    close(C.values(), want, product_bound(want, mag, dtype), f"{M}x{N}x{K}", dtype)


@pytest.mark.parametrize("K", [1, 15, 16, 17, 48, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 300, 512, 777, 1024, 1500, 2049])
@pytest.mark.parametrize("M", [1, 5, 16, 17, 32, 33, 64, 65, 130])
def test_inner_sizes(M, K):
    check(M, 70, K, "bf16", bias=True)


@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 7, 8, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 200, 333])
@pytest.mark.parametrize("M", [1, 16, 40, 64, 100, 150])
def test_columns(M, N):
    check(M, N, 96, "fp16", bias=True, ldc=N + 3, shift=1)


@pytest.mark.parametrize("M,N,K", [(128, 128, 128), (129, 257, 200), (200, 300, 1000), (256, 2048, 64), (300, 4000, 130),
                                   (1000, 1000, 100), (1025, 2050, 80), (2048, 2048, 144), (2500, 1700, 300), (70, 5000, 3000),
                                   (4096, 300, 256), (33, 9000, 500), (8, 20000, 70), (513, 1281, 4100)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_products(dtype, M, N, K):
    check(M, N, K, dtype)


@pytest.mark.parametrize("M,N,K,bias", [(4096, 4096, 512, False), (4000, 4090, 700, True), (16384, 1030, 400, False),
                                        (3900, 8200, 127, True), (8200, 4097, 40, False), (12000, 1500, 1300, True)])
def test_large_tiles(M, N, K, bias):
    """Enough 256 x 256 tiles for every compute unit, whole and ragged."""
    check(M, N, K, "bf16", bias=bias, ldc=N + 1, shift=1)


@pytest.mark.parametrize("M,N,K", [(16, 256, 16384), (1, 1, 8192), (5, 130, 8200), (40, 300, 9001), (64, 1027, 12288),
                                   (128, 1000, 8177), (33, 18, 131071)])
@pytest.mark.parametrize("bias", [False, True])
def test_inner_sizes_that_are_split(M, N, K, bias):
    assert fo.int8_workspace_bytes(M, N, K) > 0
    check(M, N, K, "fp16", bias=bias, ldc=N + 5)


@pytest.mark.parametrize("M,N,K,bias,ldc", [(5000, 5000, 1000, True, None), (8200, 4097, 1090, False, 4101), (16384, 2304, 2048, True, None),
                                            (2304, 16384, 2047, False, 16392)])
def test_tiles_one_after_another(M, N, K, bias, ldc):
    """Two or three tiles of 256 x 256 to a workgroup, whole ones and ends of rows and columns."""
    check(M, N, K, "bf16", bias=bias, ldc=ldc)


@pytest.mark.parametrize("M,N,K,bias", [(70, 9000, 100, True), (129, 8200, 40, False), (333, 2881, 1985, True), (513, 2050, 1300, False),
                                        (1000, 1100, 16, True), (128, 16384, 260, False), (33, 4500, 100, False), (64, 8192, 16, True), (100, 3001, 1000, True),
                                        (257, 1500, 700, False), (64, 4200, 32768, True), (100, 16500, 8192, True)])
def test_blocks_of_two_to_one(M, N, K, bias):
    """Blocks of 128 rows and 64 columns, and of 64 and 32; the last ones' weights past the caches' keeping."""
    check(M, N, K, "bf16", bias=bias, ldc=N + 2)
    check(M, N, K, "fp16", bias=not bias, lda=row_bytes(K) + 32)


@pytest.mark.parametrize("M", [7, 64])
def test_weights_past_the_caches(M):
    """More than 128 MiB of weights, in lines of their own, under few rows; and the same of experts."""
    check(M, 16500, 8192, "bf16", bias=True)
    Experts(M, 2, 33, 1000, 4096, "bf16", True, bias=True).check()


@pytest.mark.parametrize("M", [3, 20, 50, 90, 400])
def test_rows_apart(M):
    """Strides of all three matrices, guards between their rows (the codes' are no zeros)."""
    for K in (40, 64, 300):
        check(M, 130, K, "bf16", lda=row_bytes(K) + 16, ldb=row_bytes(K) + 48, ldc=150, shift=5)


@pytest.mark.parametrize("M", [2, 30, 60, 200])
def test_no_inner_values_leave_the_bias(M):
    torch = torch_mod()
    N, dtype = 50, "bf16"
    bias = to_dtype(np.random.default_rng(1).normal(size=N), dtype)
    for b, want in ((bias, bias), (None, np.zeros(N))):
        C = Mat(M, N, dtype)
        fo.int8_product(None, torch.ones(M, device="cuda"), None, torch.ones(N, device="cuda"), C.t, M, N, 0, dtype,
                        bias=vec(b, dtype), workspace=workspace(M, N, 0))
        np.testing.assert_array_equal(C.values(), np.broadcast_to(want, (M, N)))


@pytest.mark.parametrize("M", [1, 40, 200])
def test_the_longest_sums_are_exact(M):
    """All codes -128, or 127: the largest sums of 131071 products, 2^31 - 2^14 and less. Scales 1 / sum: c = 1."""
    K, N = 131071, 20
    for code in (-128, 127):
        a, b = np.full((M, K), code, np.int8), np.full((N, K), code, np.int8)
        b[1] = -1 - b[1] if code == -128 else -b[1]
        s = np.float32(2.0 ** -31)
        C = run(a, np.full(M, s), b, np.ones(N, np.float32), None, "fp16")
        want, mag = ref.product(a, np.full(M, s), b, np.ones(N, np.float32))
        close(C.values(), want, product_bound(want, mag, "fp16"), "longest", "fp16")


@pytest.mark.parametrize("M", [4, 40, 200])
def test_scales_at_the_edges(M):
    """Scales of zero, of NaN (a spoiled row), large beside small; results past the type's range."""
    rng = np.random.default_rng(3)
    N, K = 24, 80
    a, b = codes(rng, M, K), codes(rng, N, K)
    sa, sb = np.ones(M, np.float32), np.ones(N, np.float32)
    sa[0], sa[1], sa[2] = 0.0, np.nan, 1e30
    sb[3], sb[4], sb[5] = 0.0, 1e-30, 2.0
    C = run(a, sa, b, sb, None, "fp16")
    want, mag = ref.product(a, sa, b, sb)
    close(C.values(), want, product_bound(want, mag, "fp16"), "scales", "fp16")
    assert np.isnan(C.values()[1]).all() and (C.values()[0] == 0).all()


# ---- experts ------------------------------------------------------------------

class Experts:
    def __init__(self, T, K, E, N, H, dtype, gather, align=1, drop=0.0, bias=False, seed=0, busy=None, lda=None, ldb=None, ldc=None):
        torch = torch_mod()
        rng = np.random.default_rng(seed + T + E + N)
        ids = np.argsort(rng.normal(size=(T, E)) + (0 if busy is None else 9 * np.isin(np.arange(E), busy)), axis=1)[:, ::-1][:, :K]
        ids = np.where(rng.random((T, K)) < drop, -1, ids).astype(np.int32)
        self.offsets, self.counts, _, pairs = rowref.route_sort(ids, E, align)
        self.capacity = fo.route_capacity(T, K, E, align)
        self.pair_of = np.full(self.capacity, 12345, np.int32)        # behind the last row: as it was
        self.pair_of[:len(pairs)] = pairs
        rows = T if gather else self.capacity
        self.a, self.sa = codes(rng, rows, H), scales(rng, rows)
        self.b, self.sb = codes(rng, E, N, H), scales(rng, E, N)
        self.bias = to_dtype(rng.normal(size=(E, N)), dtype) if bias else None
        self.gather, self.K, self.dtype = gather, K, dtype
        A, B = Codes(rows, H, lda, values=self.a), Codes(E * N, H, ldb, values=self.b.reshape(E * N, H))
        self.C = Mat(self.capacity, N, dtype, ldc)
        off, cnt = dev(self.offsets.astype(np.int32)), dev(self.counts.astype(np.int32))
        fo.int8_experts(A.whole, dev(self.sa), B.whole, dev(self.sb), self.C.t, N, H, E, dtype, self.capacity, off, cnt, rows,
                        pair_of=dev(self.pair_of) if gather else None, choices=K, bias=vec(self.bias, dtype))
        torch.cuda.synchronize()

    def check(self):
        want = ref.experts(self.a, self.sa, self.b, self.sb, self.offsets, self.counts, self.capacity,
                           self.pair_of if self.gather else None, self.K, self.bias)
        assert self.C.guards_stand(list(want))
        if want:
            got = self.C.values()[list(want)]
            v, mag = (np.array([w[i] for w in want.values()]) for i in (0, 1))
            close(got, v, product_bound(v, mag, self.dtype), "experts", self.dtype)


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("T,K,E,N,H", [(1, 1, 1, 5, 16), (1, 8, 256, 40, 70), (16, 8, 256, 33, 130), (5, 2, 3, 64, 64),
                                       (40, 4, 8, 100, 200), (100, 2, 5, 130, 96), (300, 4, 16, 70, 48), (64, 8, 8, 17, 300),
                                       (700, 1, 4, 150, 100), (33, 3, 1000, 20, 32), (2000, 2, 60, 48, 40)])
def test_experts(T, K, E, N, H, gather):
    Experts(T, K, E, N, H, "bf16", gather, bias=True).check()


@pytest.mark.parametrize("align,drop", [(64, 0.0), (16, 0.3), (256, 0.1), (1, 1.0), (7, 0.5)])
@pytest.mark.parametrize("gather", [True, False])
def test_experts_padding_and_dropped(align, drop, gather):
    """Padding rows, and those behind the last, stay as they were; nothing at all where every choice is dropped."""
    for T, E in ((3, 4), (60, 8), (500, 4)):
        Experts(T, 2, E, 40, 72, "fp16", gather, align, drop).check()


@pytest.mark.parametrize("T", [10, 130, 600])
def test_one_busy_expert(T):
    """Every token to the same experts, the others empty: many blocks of rows where few were the average."""
    Experts(T, 1, 64, 40, 80, "bf16", True, busy=[63]).check()
    Experts(T, 1, 130, 40, 80, "bf16", False, busy=[0], align=64).check()
    Experts(T, 2, 100, 40, 80, "bf16", True, busy=[17, 70]).check()


@pytest.mark.parametrize("T,K,E,N,H,gather", [(4096, 2, 4, 2048, 512, True), (3000, 2, 3, 2990, 600, False), (2500, 2, 8, 3001, 300, True),
                                              (6000, 4, 30, 700, 200, True)])
def test_experts_large_tiles(T, K, E, N, H, gather):
    Experts(T, K, E, N, H, "bf16", gather, align=64, drop=0.05, bias=True).check()


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("N,H,dtype", [(1280, 1024, "bf16"), (1165, 1100, "fp16"), (1408, 1170, "bf16")])
def test_experts_of_unequal_tiles(N, H, dtype, gather):
    """More tiles of 256 x 256 than compute units, whole ones, halves and ends in turn; gaps between the experts'
    rows, rows without a token."""
    rng = np.random.default_rng(N)
    counts = np.array([512, 0, 1, 100, 128, 129, 256, 257, 300, 511, 0, 512, 600, 1000, 2000, 2500, 3333, 640, 17, 900, 768, 1100])
    gaps = rng.integers(0, 4, len(counts) + 1)
    offsets = (gaps[-1] + np.concatenate([[0], np.cumsum(counts + gaps[:-1])])).astype(np.int32)
    E, choices, cap = len(counts), 3, int(offsets[-1]) + 5
    T = cap // choices if gather else cap - 40          # (the last rows are of rows of a that are not there)
    pairs = rng.integers(0, T * choices, cap).astype(np.int32)
    pairs[::50] = -1
    pairs[7::300] = T * choices + 2
    a, sa, b, sb = codes(rng, T, H), scales(rng, T), codes(rng, E, N, H), scales(rng, E, N)
    bias = to_dtype(rng.normal(size=(E, N)), dtype)
    C = Mat(cap, N, dtype)
    counts = counts.astype(np.int32)
    fo.int8_experts(Codes(T, H, values=a).whole, dev(sa), Codes(E * N, H, values=b.reshape(E * N, H)).whole, dev(sb), C.t, N, H, E,
                    dtype, cap, dev(offsets), dev(counts), T, pair_of=dev(pairs) if gather else None, choices=choices,
                    bias=vec(bias, dtype))
    want = ref.experts(a, sa, b, sb, offsets, counts, cap, pairs if gather else None, choices, bias)
    assert C.guards_stand(list(want))
    v, mag = (np.array([w[i] for w in want.values()]) for i in (0, 1))
    close(C.values()[list(want)], v, product_bound(v, mag, dtype), "unequal tiles", dtype)
    bits = C.raw.cpu().numpy()[:cap * N].reshape(cap, N)
    left = np.setdiff1d(np.arange(cap), list(want))
    assert len(left) > 30 and (bits[left] == GUARD).all()


@pytest.mark.parametrize("H", [512, 600, 760])
@pytest.mark.parametrize("gather", [True, False])
def test_experts_short_sums_in_tiles(H, gather):
    Experts(4096, 2, 8, 4608, H, "fp16", gather, drop=0.01).check()


def test_a_thousand_experts_in_tiles():
    """As many experts as there may be, with a tile's rows each."""
    torch = torch_mod()
    rng = np.random.default_rng(8)
    E, N, H, dtype = 1024, 130, 300, "bf16"
    counts = rng.integers(100, 240, E).astype(np.int32)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    cap = int(offsets[-1])
    a, sa, b, sb = codes(rng, cap, H), scales(rng, cap), codes(rng, E, N, H), scales(rng, E, N)
    C = Mat(cap, N, dtype)
    fo.int8_experts(Codes(cap, H, values=a).whole, dev(sa), Codes(E * N, H, values=b.reshape(E * N, H)).whole, dev(sb), C.t, N, H, E,
                    dtype, cap, dev(offsets), dev(counts), cap)
    torch.cuda.synchronize()
    got = C.values()
    for e in rng.choice(E, 60, replace=False):
        rows = slice(offsets[e], offsets[e + 1])
        want, mag = ref.product(a[rows], sa[rows], b[e], sb[e])
        close(got[rows], want, product_bound(want, mag, dtype), f"expert {e}", dtype)
    assert C.guards_stand()


@pytest.mark.parametrize("H", [16, 100, 500, 1500])
def test_experts_several_blocks_to_a_workgroup(H):
    """Short sums and many columns."""
    Experts(40, 4, 60, 2300, H, "fp16", True, bias=True).check()
    Experts(1000, 2, 16, 2300, min(H, 500), "bf16", False).check()


@pytest.mark.parametrize("T,K,E,N,H", [(200, 4, 160, 2500, 40), (200, 4, 160, 2530, 300), (200, 4, 160, 2499, 900), (750, 4, 60, 4500, 200),
                                       (750, 4, 60, 4555, 500), (16, 8, 256, 1100, 130), (500, 4, 200, 64, 70)])
def test_experts_many_blocks(T, K, E, N, H):
    """Several blocks to a workgroup, of 64 and of 128 columns, the last one past the columns' end; blocks of 128
    for a few rows; of 64 for 64 columns."""
    Experts(T, K, E, N, H, "bf16", True, bias=True, drop=0.1).check()
    Experts(T, K, E, N, H, "fp16", False).check()


def test_experts_rows_apart():
    Experts(50, 2, 6, 37, 100, "bf16", True, lda=128, ldb=160, ldc=45).check()
    Experts(300, 2, 3, 150, 100, "bf16", False, lda=144, ldb=128, ldc=151).check()


@pytest.mark.parametrize("T", [4, 60, 300])
def test_rows_without_a_token_are_left(T):
    """Pairs outside the tokens, ranges past the capacity or before it: those rows are not written, nothing faults."""
    torch = torch_mod()
    rng = np.random.default_rng(T)
    K, E, N, H, dtype = 2, 4, 24, 64, "bf16"
    cap = T * K
    a, sa, b, sb = codes(rng, T, H), scales(rng, T), codes(rng, E, N, H), scales(rng, E, N)
    pairs = rng.permutation(cap).astype(np.int32)
    pairs[::5] = -1 - pairs[::5]
    pairs[1::7] += K * T
    counts = np.array([cap // 4, cap // 4, cap, 3], np.int32)         # the third runs past the end
    offsets = np.array([0, cap // 4, cap // 2, -2, 0], np.int32)      # the fourth begins before the start
    C = Mat(cap, N, dtype)
    fo.int8_experts(Codes(T, H, values=a).whole, dev(sa), Codes(E * N, H, values=b.reshape(E * N, H)).whole, dev(sb), C.t, N, H, E,
                    dtype, cap, dev(offsets), dev(counts), T, pair_of=dev(pairs), choices=K)
    want = ref.experts(a, sa, b, sb, offsets[:3], counts[:3], cap, pairs, K)
    assert C.guards_stand(list(want))
    v, mag = (np.array([w[i] for w in want.values()]) for i in (0, 1))
    close(C.values()[list(want)], v, product_bound(v, mag, dtype), "pairs", dtype)
    bits = C.raw.cpu().numpy()[:cap * N].reshape(cap, N)
    left = [r for r in range(cap) if r not in want]
    assert left and (bits[left] == GUARD).all()
    torch.cuda.synchronize()


def test_equal_calls_give_equal_bits_in_every_order_of_rows():
    """A row's result does not depend on the rows beside it (the sums are exact): alone, among few, among many."""
    rng = np.random.default_rng(4)
    N, K, dtype = 200, 700, "fp16"
    a, b, sa, sb = codes(rng, 600, K), codes(rng, N, K), scales(rng, 600), scales(rng, N)
    many = run(a, sa, b, sb, None, dtype).bits()
    for M in (1, 16, 20, 33, 64, 65, 200):
        np.testing.assert_array_equal(run(a[:M], sa[:M], b, sb, None, dtype).bits(), many[:M])
