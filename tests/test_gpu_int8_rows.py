"""Rows in 8-bit integers and the RMS norm of a sum, forward and backward, against the
64-bit reference: every form of the kernels, odd lengths, strides and offsets, rows of
zeros, infinities and NaN, in place, one row and many."""
import numpy as np
import pytest

import oracle
import paper_2504_19519_amd as fo
from gpu_util import torch_mod
from int8_util import (RSTD, Codes, F32, check_grads, check_norm_codes, check_quantized, f32_vec, kept_sum, to_dtype)
from oracle import int8ops as ref
from rowops_util import Mat, close, rounded, torch_dtype

pytestmark = pytest.mark.gpu
DTYPES = ["fp16", "bf16"]
# lengths of every form: threads to a row, chunks to a thread, and ends of each kind
LENGTHS = [1, 2, 5, 7, 8, 9, 15, 16, 17, 63, 64, 65, 100, 128, 129, 250, 256, 257, 511, 512, 513, 1000, 1024, 1030, 2047,
           2048, 2051, 4096, 4097, 5000, 6144, 6150, 8192, 8193, 12288, 12295, 16384, 16385, 20001, 24576, 24580, 32761, 32768]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = torch_mod()
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    fo.lib()
    yield
    torch.cuda.synchronize()


def stream_values(rng, M, N, dtype):
    """Rows of uneven size, columns too."""
    return to_dtype(rng.normal(size=(M, N)) * np.exp2(rng.integers(-6, 6, (M, 1))) * rng.uniform(0.2, 3.0, N), dtype)


def tensor(values):
    return torch_mod().as_tensor(np.asarray(values))


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def vec(values, dtype):
    return tensor(values).to("cuda").to(torch_dtype(dtype))


def quantize(x, dtype, ld=None, shift=0, ldc=None):
    M, N = x.shape
    X, C, s = Mat(M, N, dtype, ld, shift, tensor(x)), Codes(M, N, ldc), f32_vec(M + 1)
    fo.quantize_rows(X.t, C.whole, s, M, N, dtype)
    assert C.guards_stand() and C.rest_is_zero() and float(s[M]) == -7.0 and X.guards_stand()
    return C.values(), s[:M].cpu().numpy()


@pytest.mark.parametrize("N", LENGTHS + [32769, 40000, 70001])
@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_lengths(dtype, N):
    rng = np.random.default_rng(N)
    for M in (1, 5):
        x = stream_values(rng, M, N, dtype)
        codes, scales = quantize(x, dtype, ld=N + 3, shift=1, ldc=-(-N // 16) * 16 + 16)
        check_quantized(codes, scales, x, f"{M}x{N}")


@pytest.mark.parametrize("M,N", [(3000, 40), (700, 64), (9000, 200), (5000, 1000), (2100, 2304), (4200, 33), (600, 5003)])
def test_quantize_many_rows(M, N):
    rng = np.random.default_rng(M)
    x = stream_values(rng, M, N, "bf16")
    check_quantized(*quantize(x, "bf16"), x, f"{M}x{N}")


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_ties_go_to_even(dtype):
    """Values half way between two codes: m = 127 * 2^j and x = (n + 1/2) * 2^j; and every value of some magnitudes m."""
    rows = []
    for j in (-10, 0, 6):
        row = np.zeros(256)
        row[:254] = (np.arange(-127, 127) + 0.5) * 2.0 ** j
        row[255] = 127 * 2.0 ** j
        rows.append(row)
    x = np.array(rows)
    assert (to_dtype(x, dtype) == x).all()
    codes, scales = quantize(x, dtype)
    check_quantized(codes, scales, x, "ties")
    assert (codes[:, :254] % 2 == 0).all()
    bits = np.arange(0x3C00, 0x4000, 4, dtype=np.uint16) if dtype == "fp16" else np.arange(0x3F80, 0x4000, dtype=np.uint16)
    v = oracle.decode(bits, dtype).astype(np.float64)
    x = np.concatenate([v[:, None], np.where(v[None] <= v[:, None], v[None], v[None] / 4)], axis=1)
    check_quantized(*quantize(x, dtype), x, "every magnitude")


@pytest.mark.parametrize("N", [3, 64, 300, 4100, 40000])
@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_zeros_extremes_and_not_numbers(dtype, N):
    top = 65504.0 if dtype == "fp16" else float(oracle.decode(np.array([0x7F7F], np.uint16), "bf16")[0])
    low = 2.0 ** -24 if dtype == "fp16" else 2.0 ** -133
    x = np.ones((9, N))
    x[0] = 0.0
    x[1] = -0.0
    x[2] = top
    x[2, N // 2] = -top
    x[3] = low
    x[4] = np.where(np.arange(N) % 2 == 0, low, 3 * low)
    x[5, N - 1] = np.inf
    x[6, 0] = -np.inf
    x[7, N // 2] = np.nan
    codes, scales = quantize(x, dtype)
    want, s = ref.quantize(x)
    np.testing.assert_array_equal(codes, want)
    with np.errstate(invalid="ignore"):
        m = np.abs(x).max(axis=1).astype(np.float32) / np.float32(127)
    np.testing.assert_array_equal(scales, np.where(np.isfinite(s), m, np.float32(np.nan)))
    assert np.isnan(scales[[5, 6, 7]]).all() and (codes[5:8] == 0).all() and scales[0] == 0


class Norm:
    """One forward pass: what it read and what it wrote."""

    def __init__(self, x, r, gamma, dtype, eps=1e-6, want=("h", "y", "rstd", "codes"), ld=0, shift=0):
        M, N = x.shape
        self.M, self.N, self.dtype, self.eps, self.gamma = M, N, dtype, eps, gamma
        mat = lambda v=None: Mat(M, N, dtype, N + ld, shift, None if v is None else tensor(v))
        X, R = mat(x), None if r is None else mat(r)
        self.h, self.y = (mat() if k in want else None for k in ("h", "y"))
        self.rstd = f32_vec(M + 1) if "rstd" in want else None
        self.codes, self.scales = (Codes(M, N), f32_vec(M + 1)) if "codes" in want else (None, None)
        t = lambda m: None if m is None else m.t
        fo.norm_add_forward(X.t, t(R), None if gamma is None else vec(gamma, dtype), t(self.h), t(self.y), M, N, dtype, eps,
                            rstd=self.rstd, codes=None if self.codes is None else self.codes.whole, scales=self.scales)
        torch_mod().cuda.synchronize()
        self.want_h = kept_sum(x, r, dtype)

    def check(self, what):
        h, dtype, M = self.want_h, self.dtype, self.M
        rstd, y = ref.norm_add(h, self.gamma, self.eps)
        if self.h is not None:
            np.testing.assert_array_equal(self.h.values(), h, err_msg=what)
            assert self.h.guards_stand()
        if self.rstd is not None:
            close(self.rstd[:M].cpu().numpy(), rstd, rstd * RSTD, what + " rstd")
            assert float(self.rstd[M]) == -7.0
        if self.y is not None:
            close(self.y.values(), y, rounded(y, dtype, np.abs(y) * (RSTD + 2 * F32)), what + " y", dtype)
            assert self.y.guards_stand()
        if self.codes is not None:
            check_norm_codes(self.codes.values(), self.scales[:M].cpu().numpy(), h, self.gamma, rstd, what)
            assert self.codes.guards_stand() and self.codes.rest_is_zero() and float(self.scales[M]) == -7.0


def inputs(rng, M, N, dtype):
    return (to_dtype(rng.normal(size=(M, N)), dtype), stream_values(rng, M, N, dtype), to_dtype(rng.uniform(0.5, 1.5, N), dtype))


@pytest.mark.parametrize("N", LENGTHS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_add_lengths(dtype, N):
    rng = np.random.default_rng(N)
    for M in (1, 6):
        x, r, gamma = inputs(rng, M, N, dtype)
        Norm(x, r, gamma, dtype, ld=5, shift=3).check(f"{M}x{N}")


@pytest.mark.parametrize("want", [("y",), ("codes",), ("h", "codes"), ("h", "y", "rstd"), ("y", "codes", "rstd")])
@pytest.mark.parametrize("residual,gamma", [(True, False), (False, True), (False, False)])
def test_norm_add_any_outputs(want, residual, gamma):
    rng = np.random.default_rng(3)
    for M, N in ((4, 100), (3, 2500)):
        x, r, g = inputs(rng, M, N, "bf16")
        Norm(x, r if residual else None, g if gamma else None, "bf16", want=want).check(str(want))


@pytest.mark.parametrize("M,N", [(5000, 60), (5000, 130), (3000, 300), (4200, 1000), (3000, 2048), (2100, 2304), (1100, 6000),
                                 (700, 9000)])
def test_norm_add_many_rows(M, N):
    rng = np.random.default_rng(M + N)
    x, r, gamma = inputs(rng, M, N, "fp16")
    Norm(x, r, gamma, "fp16").check(f"{M}x{N}")


@pytest.mark.parametrize("N", [6, 60, 1000, 4100, 20000])
@pytest.mark.parametrize("which", ["hx", "hr", "yx", "yr"])
def test_norm_add_in_place(which, N):
    """h or y written over x or the residual."""
    rng = np.random.default_rng(N)
    M, dtype = 7, "bf16"
    x, r, gamma = inputs(rng, M, N, dtype)
    X, R, out = (Mat(M, N, dtype, N + 2, 1, v) for v in (tensor(x), tensor(r), None))
    over = X if which[1] == "x" else R
    h, y = (over, out) if which[0] == "h" else (out, over)
    fo.norm_add_forward(X.t, R.t, vec(gamma, dtype), h.t, y.t, M, N, dtype, 1e-6)
    want_h = kept_sum(x, r, dtype)
    rstd, want = ref.norm_add(want_h, gamma, 1e-6)
    np.testing.assert_array_equal(h.values(), want_h)
    close(y.values(), want, rounded(want, dtype, np.abs(want) * (RSTD + 2 * F32)), which, dtype)
    assert h.guards_stand() and y.guards_stand()


def test_norm_add_zeros_and_not_numbers():
    M, N, dtype = 5, 700, "bf16"
    x, r = np.zeros((M, N)), np.ones((M, N))
    r[0] = 0.0                       # a row of zeros: y = 0
    x[1], r[1] = 3.0, -3.0           # which cancel
    r[2, 5] = np.inf
    r[3, 699] = np.nan
    X, R, H, Y, C, s = Mat(M, N, dtype, values=tensor(x)), Mat(M, N, dtype, values=tensor(r)), Mat(M, N, dtype), Mat(M, N, dtype), \
        Codes(M, N), f32_vec(M)
    fo.norm_add_forward(X.t, R.t, None, H.t, Y.t, M, N, dtype, 1e-6, codes=C.whole, scales=s)
    y, codes, scales = Y.values(), C.values(), s.cpu().numpy()
    assert (y[:2] == 0).all() and (codes[:2] == 0).all() and (scales[:2] == 0).all()
    assert np.isnan(y[2, 5]) and (np.delete(y[2], 5) == 0).all() and np.isnan(y[3]).all()
    assert np.isnan(scales[2]) and np.isnan(scales[3]) and (codes[2:4] == 0).all()
    assert (codes[4] == 127).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_add_large_and_small_values(dtype):
    """Values whose squares are far from 1, and gammas too."""
    rng = np.random.default_rng(8)
    for N in (48, 3000):
        for scale, g in ((2.0 ** -12, 1.0), (2.0 ** 12, 2.0 ** 3), (1.0, 2.0 ** -9)) if dtype == "fp16" else \
                ((2.0 ** -70, 2.0 ** 40), (2.0 ** 58, 2.0 ** -50), (1.0, 2.0 ** -100)):
            x, r, gamma = (to_dtype(v, dtype) for v in (rng.uniform(-1, 1, (3, N)) * scale, rng.uniform(-1, 1, (3, N)) * scale,
                                                         rng.uniform(0.5, 1, N) * g))
            Norm(x, r, gamma, dtype, eps=0.0).check(f"{N} {scale} {g}") if dtype == "bf16" and scale > 1e-10 else \
                Norm(x, r, gamma, dtype, eps=1e-30 if dtype == "bf16" else 1e-9).check(f"{N} {scale} {g}")


# ---- backward ---------------------------------------------------------------

def backward(M, N, dtype, seed, dh=True, gamma=True, want=("dx", "dgamma"), ld=0, shift=0, over=None):
    torch = torch_mod()
    rng = np.random.default_rng(seed)
    dyv, dhv, hv = to_dtype(rng.normal(size=(M, N)), dtype), to_dtype(rng.normal(size=(M, N)), dtype), stream_values(rng, M, N, dtype)
    gv = to_dtype(rng.uniform(0.5, 1.5, N), dtype)
    rstd = (1.0 / np.sqrt((hv * hv).mean(axis=1) + 1e-6)).astype(np.float32)
    mat = lambda v=None: Mat(M, N, dtype, N + ld, shift, None if v is None else tensor(v))
    at = {"dy": mat(dyv), "dh": mat(dhv) if dh else None, "h": mat(hv)}
    dx = at[over] if over else mat() if "dx" in want else None
    dgamma = f32_vec(N + 1) if "dgamma" in want else None
    work = torch.full((fo.norm_workspace_bytes(M, N),), 0xFF, dtype=torch.uint8, device="cuda")
    fo.norm_add_backward(at["dy"].t, at["dh"].t if dh else None, at["h"].t, vec(gv, dtype) if gamma else None,
                         tensor(rstd).cuda(), dx.t if dx else None, dgamma, M, N, dtype, work)
    check_grads(dx.values() if dx else None, None if dgamma is None else dgamma[:N].cpu().numpy(), dyv, dhv if dh else None, hv,
                gv if gamma else None, rstd.astype(np.float64), dtype, f"{M}x{N}")
    assert dx is None or dx.guards_stand()
    assert dgamma is None or float(dgamma[N]) == -7.0


@pytest.mark.parametrize("N", LENGTHS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_add_backward_lengths(dtype, N):
    for M in (1, 6):
        backward(M, N, dtype, N + M, ld=3, shift=1)


@pytest.mark.parametrize("M,N", [(5000, 8), (40000, 40), (9000, 100), (9000, 200), (6000, 300), (5000, 700), (3000, 1500),
                                 (2100, 2304), (1030, 4096), (800, 6001), (600, 10000), (520, 14000), (300, 20004)])
def test_norm_add_backward_many_rows(M, N):
    backward(M, N, "bf16", M)


@pytest.mark.parametrize("M", [255, 256, 257, 511, 512, 513, 767, 1024, 1025])
def test_norm_add_backward_rows_around_the_rounds(M):
    for N in (130, 1000, 4096):
        backward(M, N, "fp16", M)


@pytest.mark.parametrize("kw", [dict(dh=False), dict(gamma=False), dict(want=("dx",)), dict(want=("dgamma",)),
                                dict(dh=False, gamma=False)])
def test_norm_add_backward_without(kw):
    for M, N in ((5, 100), (300, 3000), (9, 20000)):
        backward(M, N, "bf16", 11, **kw)


@pytest.mark.parametrize("over", ["dy", "dh", "h"])
def test_norm_add_backward_in_place(over):
    for M, N in ((5, 6), (300, 60), (300, 1001), (40, 4099), (30, 9001), (20, 20005)):
        backward(M, N, "fp16", 12, over=over, ld=1)


def test_norm_add_gradients_against_differences():
    """The GPU's gradients against differences of the reference's own forward pass in 64 bits."""
    M, N, dtype, eps, d = 3, 20, "bf16", 1e-3, 1e-5
    rng = np.random.default_rng(5)
    x, r, gamma = inputs(rng, M, N, dtype)
    dyv, dhv = to_dtype(rng.normal(size=(M, N)), dtype), to_dtype(rng.normal(size=(M, N)), dtype)
    n = Norm(x, r, gamma, dtype, eps, want=("h", "y", "rstd"))
    h = n.h.values()

    def loss(h, gamma):
        return (ref.norm_add(h, gamma, eps)[1] * dyv).sum() + (h * dhv).sum()
    dx, dgamma = Mat(M, N, dtype), f32_vec(N)
    work = torch_mod().empty(fo.norm_workspace_bytes(M, N), dtype=torch_mod().uint8, device="cuda")
    fo.norm_add_backward(Mat(M, N, dtype, values=tensor(dyv)).t, Mat(M, N, dtype, values=tensor(dhv)).t, n.h.t, vec(gamma, dtype),
                         n.rstd, dx.t, dgamma, M, N, dtype, work)
    got = dx.values()
    for i in np.ndindex(M, N):
        hi, lo = h.copy(), h.copy()
        hi[i] += d
        lo[i] -= d
        diff = (loss(hi, gamma) - loss(lo, gamma)) / (2 * d)
        # half a step of bf16, the kernel's 32 bits, the differences' own 1e-6
        assert abs(got[i] - diff) <= 2.0 ** -8 * abs(diff) + 1e-5, i
    for j in range(N):
        hi, lo = gamma.copy(), gamma.copy()
        hi[j] += d
        lo[j] -= d
        assert abs(float(dgamma[j]) - (loss(h, hi) - loss(h, lo)) / (2 * d)) <= 1e-5


def test_equal_calls_give_equal_bits():
    torch = torch_mod()
    M, N, dtype = 1500, 2880, "bf16"
    rng = np.random.default_rng(2)
    dy, dh, h = (Mat(M, N, dtype, values=tensor(rng.normal(size=(M, N)))) for _ in range(3))
    rstd, gamma = torch.rand(M, device="cuda") + 0.5, vec(rng.uniform(0.5, 1.5, N), dtype)
    work = torch.empty(fo.norm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
    got = []
    for fill in (0x00, 0xFF, 0x7F):
        work.fill_(fill)
        dx, dgamma = Mat(M, N, dtype), f32_vec(N)
        fo.norm_add_backward(dy.t, dh.t, h.t, gamma, rstd, dx.t, dgamma, M, N, dtype, work)
        got.append((dx.bits(), dgamma.cpu().numpy()))
    for a, b in got[1:]:
        np.testing.assert_array_equal(a, got[0][0])
        np.testing.assert_array_equal(b, got[0][1])


def test_no_rows_zero_the_sums():
    dgamma = f32_vec(40)
    fo.norm_add_backward(None, None, None, None, None, None, dgamma, 0, 40, "bf16", None)
    assert (dgamma == 0).all()
    fo.quantize_rows(None, None, None, 0, 40, "bf16")
    fo.norm_add_forward(None, None, None, None, None, 0, 40, "bf16")


@pytest.mark.parametrize("M,N", [(300000, 57), (140000, 121), (70000, 250), (35000, 500), (17000, 1001), (9000, 2000), (4200, 4099),
                                 (2900, 6000), (2100, 8190), (1500, 12001), (1100, 16000), (700, 24570)])
def test_matrices_past_the_caches(M, N):
    """Sizes whose loads pass the caches by: the first, the last and some rows between against
    the reference, the sums over all rows against 64 bits on the GPU."""
    torch = torch_mod()
    assert M * N > 1 << 24
    dtype = "bf16"
    gen = torch.Generator(device="cuda").manual_seed(M)
    x, r, dy, dh = (torch.randn(M, N, generator=gen, device="cuda").bfloat16() for _ in range(4))
    gamma = (torch.rand(N, generator=gen, device="cuda") + 0.5).bfloat16()
    at = np.unique(np.concatenate([np.arange(20), np.arange(M - 20, M), np.random.default_rng(M).integers(0, M, 40)]))
    some = lambda t: t[torch.as_tensor(at).cuda()].double().cpu().numpy()
    codes, scales = torch.zeros(M, fo.int8_row_bytes(N), dtype=torch.int8, device="cuda"), f32_vec(M)
    fo.quantize_rows(x, codes, scales, M, N, dtype)
    check_quantized(some(codes)[:, :N].astype(np.int8), some(scales).astype(np.float32), some(x), "quantize")
    assert not bool(codes[:, N:].any())
    h, y, dx = (torch.empty_like(x) for _ in range(3))
    rstd, dgamma = f32_vec(M), f32_vec(N)
    fo.norm_add_forward(x, r, gamma, h, y, M, N, dtype, 1e-6, rstd=rstd, codes=codes, scales=scales)
    want_h = kept_sum(some(x), some(r), dtype)
    np.testing.assert_array_equal(some(h), want_h)
    g = host(gamma)
    want_r, want = ref.norm_add(want_h, g, 1e-6)
    close(some(rstd), want_r, want_r * RSTD, "rstd")
    close(some(y), want, rounded(want, dtype, np.abs(want) * (RSTD + 2 * F32)), "y", dtype)
    check_norm_codes(some(codes)[:, :N].astype(np.int8), some(scales), want_h, g, want_r, "codes")
    work = torch.empty(fo.norm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
    fo.norm_add_backward(dy, dh, h, gamma, rstd, dx, dgamma, M, N, dtype, work)
    check_grads(some(dx), None, some(dy), some(dh), want_h, g, some(rstd), dtype, "backward")
    terms = dy.double() * h.double() * rstd.double()[:, None]
    steps = -(-M // 64) + 24 + 3
    close(dgamma.cpu().numpy(), terms.sum(0).cpu().numpy(), steps * F32 * terms.abs().sum(0).cpu().numpy(), "dgamma")
