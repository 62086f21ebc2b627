"""Layer norm / RMS norm and its backward pass on the GPU against the 64-bit
reference, through the C ABI.

Bounds. A row's sum of n products is a tree of at most 8 * 4 chunks per lane, 6
steps over a wave, 16 waves and a tail: fewer than 64 additions in a chain, so its
error is below 64 * 2^-24 of the sum of magnitudes; S = 2^-18. Forward: the mean is
off by S * mean|x|, the variance (differences from that mean) by 2 S of itself plus the
mean's error squared, so y's error before rounding is within
|gamma| (|h| 2 S + rstd S mean|x|) + 2^-22 (|gamma h| + |beta|). Backward: the
statistics are inputs; h is off by 2^-23 |h| + 2^-23, the two means by 2 S of their
sums of magnitudes. A column's sum over rows has fewer than M + 64 additions in a chain."""
import itertools

import numpy as np
import pytest

import paper_2504_19519_amd as fo
from gpu_util import say, torch_mod
from oracle import rowops as ref
from rowops_util import F32, Mat, close, rounded, torch_dtype

pytestmark = pytest.mark.gpu
S = 2.0 ** -18


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = torch_mod()
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    fo.lib()
    yield
    torch.cuda.synchronize()


def vec(values, dtype):
    torch = torch_mod()
    return torch.as_tensor(values).to(torch_dtype(dtype)).cuda()


def f32(n, fill=float("nan")):
    torch = torch_mod()
    return torch.full((max(n, 1),), fill, dtype=torch.float32, device="cuda")


def kept_of(M, N):
    torch = torch_mod()
    a, b = fo.packed_bytes(M, N)
    return torch.full((a,), 77, dtype=torch.uint8, device="cuda"), torch.full((b,), 77, dtype=torch.uint8, device="cuda")


def host(t):
    return t.detach().double().cpu().numpy()


def inputs(M, N, dtype, seed, ld=None, shift=0, affine=True):
    rng = np.random.default_rng(seed)
    torch = torch_mod()
    x = Mat(M, N, dtype, ld, shift, torch.as_tensor(rng.normal(size=(M, N)) * np.exp(rng.normal(size=N)) +
                                                    rng.normal(size=(M, 1)) * 3))
    dy = Mat(M, N, dtype, ld, shift, torch.as_tensor(rng.normal(size=(M, N))))
    gamma = vec(rng.uniform(0.5, 1.5, N), dtype) if affine else None
    beta = vec(rng.normal(size=N), dtype) if affine else None
    return x, dy, gamma, beta


def check_forward(kind, x, gamma, beta, y, mean, rstd, eps, what):
    v, g, b = x.values(), 1.0 if gamma is None else host(gamma), 0.0 if beta is None else host(beta)
    m, r = ref.norm_stats(v, kind, eps)
    want = ref.norm(v, m, r, g, b)
    mag = np.abs(v).mean(axis=1)[:, None]
    h = np.abs(v - m[:, None]) * r[:, None]
    extra = np.abs(g) * (h * 2 * S + (r[:, None] * S * mag if kind == "layer" else 0)) + 2.0 ** -22 * (np.abs(g) * h + np.abs(b))
    close(y.values(), want, rounded(want, y.dtype, extra), what + " y", y.dtype)
    assert y.guards_stand(), what
    if mean is not None:
        close(host(mean)[:len(m)], m, S * mag[:, 0] + F32 * np.abs(m), what + " mean")
    if rstd is not None:
        close(host(rstd)[:len(r)], r, r * (2 * S + (S * mag[:, 0] * r) ** 2), what + " rstd")


def check_backward(kind, fmt, x, dy, gamma, mean, rstd, dx, dgamma, dbeta, what, dy_values=None):
    v = x.values()
    if fmt != "none":
        v = ref.unpack(*ref.pack(v, fmt, x.dtype), x.N, fmt)
    d = dy.values() if dy_values is None else dy_values
    g = 1.0 if gamma is None else host(gamma)
    r = host(rstd)[:x.M]
    m = host(mean)[:x.M] if kind == "layer" else np.zeros(x.M)
    want, dg, db = ref.norm_grad(d, v, m, r, g, kind)
    h, gd = (v - m[:, None]) * r[:, None], d * g
    dh = 2.0 ** -23 * (np.abs(h) + 1)
    m1, m2 = gd.mean(axis=1, keepdims=True), (gd * h).mean(axis=1, keepdims=True)
    e1 = 2 * S * np.abs(gd).mean(axis=1, keepdims=True)
    e2 = 2 * S * (np.abs(gd * h)).mean(axis=1, keepdims=True) + (np.abs(gd) * dh).mean(axis=1, keepdims=True)
    extra = r[:, None] * (2.0 ** -22 * (np.abs(gd) + np.abs(m1) + np.abs(h * m2)) + dh * np.abs(m2) + np.abs(h) * e2 +
                          (e1 if kind == "layer" else 0))
    if dx is not None:
        close(dx.values(), want, rounded(want, dx.dtype, extra), what + " dx", dx.dtype)
        assert dx.guards_stand(), what
    n = (x.M + 64) * F32
    if dgamma is not None:
        close(host(dgamma)[:x.N], dg, n * np.abs(d * h).sum(axis=0) + (np.abs(d) * dh).sum(axis=0), what + " dgamma")
    if dbeta is not None:
        close(host(dbeta)[:x.N], db, n * np.abs(d).sum(axis=0), what + " dbeta")


def both(kind, M, N, dtype, fmt, seed, ld=None, shift=0, affine=True, eps=1e-6, given=None):
    torch = torch_mod()
    what = f"[norm] {kind} {M}x{N} {dtype} {fmt} ld={ld} shift={shift} affine={affine}"
    say(what)
    x, dy, gamma, beta = given or inputs(M, N, dtype, seed, ld, shift, affine)
    y, dx = Mat(M, N, dtype, ld, shift), Mat(M, N, dtype, ld, shift)
    mean, rstd = f32(M), f32(M)
    codes, scales = kept_of(M, N) if fmt != "none" else (None, None)
    kept = {} if fmt == "none" else dict(packed=codes, scales=scales, fmt=fmt)
    fo.norm_forward(kind, x.t, gamma, beta, y.t, M, N, dtype, eps, mean, rstd, **kept)
    torch.cuda.synchronize()
    check_forward(kind, x, gamma, beta, y, mean, rstd, eps, what)
    if fmt != "none":
        c, s = ref.pack(x.values(), fmt, dtype)
        np.testing.assert_array_equal(scales.cpu().numpy(), s.reshape(-1), err_msg=what)
        np.testing.assert_array_equal(codes.cpu().numpy(), c.reshape(-1), err_msg=what)
    dgamma, dbeta = f32(N), f32(N)
    work = torch.full((fo.norm_workspace_bytes(M, N),), 0xFF, dtype=torch.uint8, device="cuda")
    fo.norm_backward(kind, dy.t, None if kept else x.t, gamma, mean, rstd, dx.t, dgamma, dbeta, M, N, dtype, work, **kept)
    torch.cuda.synchronize()
    check_backward(kind, fmt, x, dy, gamma, mean, rstd, dx, dgamma, dbeta, what)


LENGTHS = [1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 100, 511, 512, 513, 1000, 1024, 1032, 2048, 2049, 2056, 4095, 4096, 4104, 8192,
           8193, 8200, 12288, 16384, 16385, 20000, 32767, 32768]


@pytest.mark.parametrize("N", LENGTHS)
def test_lengths(N):
    for i, (kind, dtype, fmt) in enumerate(itertools.product(["layer", "rms"], ["fp16", "bf16"], ["none", "int8", "e4m3"])):
        both(kind, 5, N, dtype, fmt, 100 + i)


@pytest.mark.parametrize("M", [1, 2, 3, 4, 6, 511, 512, 513, 1030, 2051])
@pytest.mark.parametrize("N", [40, 2049, 2304])
def test_row_counts(M, N):
    both("layer", M, N, "bf16", "none", 7)
    both("rms", M, N, "fp16", "int8", 8)


@pytest.mark.parametrize("N,ld,shift", [(64, 64, 1), (100, 101, 3), (512, 520, 8), (1000, 1999, 5), (2880, 5761, 2),
                                        (4096, 8192, 4), (9000, 9001, 7)])
def test_strides_and_alignment(N, ld, shift):
    for kind, fmt in itertools.product(["layer", "rms"], ["none", "int8", "e4m3"]):
        both(kind, 9, N, "bf16", fmt, 11, ld, shift)
    both("layer", 9, N, "fp16", "none", 12, ld, shift, affine=False)


def test_explicit_row_distances_and_raw_pointers():
    torch = torch_mod()
    M, N, ld = 6, 72, 80
    x, dy, gamma, beta = inputs(M, N, "bf16", 3, ld)
    y, dx = Mat(M, N, "bf16", ld), Mat(M, N, "bf16", ld)
    mean, rstd, dgamma, dbeta = f32(M), f32(M), f32(N), f32(N)
    work = torch.empty(fo.norm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
    fo.norm_forward("layer", x.raw, gamma, beta, y.raw.data_ptr(), M, N, "bf16", 1e-6, mean, rstd, ldx=ld, ldy=ld)
    fo.norm_backward("layer", dy.raw, x.raw.data_ptr(), gamma, mean, rstd, dx.raw, dgamma, dbeta, M, N, "bf16", work.data_ptr(),
                     lddy=ld, ldx=ld, lddx=ld)
    torch.cuda.synchronize()
    check_forward("layer", x, gamma, beta, y, mean, rstd, 1e-6, "raw")
    check_backward("layer", "none", x, dy, gamma, mean, rstd, dx, dgamma, dbeta, "raw")


@pytest.mark.parametrize("N", [96, 2052, 3000, 16400])
def test_in_place(N):
    torch = torch_mod()
    M, dtype = 7, "fp16"
    for fmt in ("none", "int8"):
        x, dy, gamma, beta = inputs(M, N, dtype, 21)
        kept = dict(zip(("packed", "scales", "fmt"), kept_of(M, N) + (fmt,))) if fmt != "none" else {}
        y, y2 = Mat(M, N, dtype), Mat(M, N, dtype, values=x.t)
        mean, rstd = f32(M), f32(M)
        fo.norm_forward("layer", x.t, gamma, beta, y.t, M, N, dtype, 1e-6, mean, rstd)
        fo.norm_forward("layer", y2.t, gamma, beta, y2.t, M, N, dtype, 1e-6, **kept)
        np.testing.assert_array_equal(y.bits(), y2.bits())
        dx, work = Mat(M, N, dtype), torch.empty(fo.norm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
        src = None if kept else x.t
        fo.norm_backward("layer", dy.t, src, gamma, mean, rstd, dx.t, None, None, M, N, dtype, work if N > 16384 else None, **kept)
        over = Mat(M, N, dtype, values=dy.t)
        fo.norm_backward("layer", over.t, src, gamma, mean, rstd, over.t, f32(N), None, M, N, dtype, work, **kept)
        np.testing.assert_array_equal(dx.bits(), over.bits())
        if not kept:
            over = Mat(M, N, dtype, values=x.t)
            fo.norm_backward("layer", dy.t, over.t, gamma, mean, rstd, over.t, None, f32(N), M, N, dtype, work)
            np.testing.assert_array_equal(dx.bits(), over.bits())


def test_parts_of_the_gradient():
    torch = torch_mod()
    M, N, dtype = 37, 520, "bf16"
    x, dy, gamma, beta = inputs(M, N, dtype, 31)
    y, mean, rstd = Mat(M, N, dtype), f32(M), f32(M)
    fo.norm_forward("rms", x.t, gamma, None, y.t, M, N, dtype, 1e-5, mean, rstd)
    torch.cuda.synchronize()
    assert (host(mean) == 0).all()                       # an RMS norm has none
    work = torch.empty(fo.norm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
    for with_dx, with_g, with_b in itertools.product([0, 1], [0, 1], [0, 1]):
        if not (with_dx or with_g or with_b):
            continue
        dx, dg, db = Mat(M, N, dtype) if with_dx else None, f32(N) if with_g else None, f32(N) if with_b else None
        fo.norm_backward("rms", dy.t, x.t, gamma, None, rstd, dx.t if dx else None, dg, db, M, N, dtype,
                         work if with_g or with_b else None)
        torch.cuda.synchronize()
        check_backward("rms", "none", x, dy, gamma, None, rstd, dx, dg, db, f"parts {with_dx}{with_g}{with_b}")


def test_wide_rows_in_parts():
    """Rows past 16384 columns: two launches, the first for dx alone."""
    torch = torch_mod()
    for M, N in ((1, 16385), (130, 20000), (70, 32768), (259, 16400)):
        for dtype, fmt in (("bf16", "none"), ("fp16", "int8"), ("bf16", "e4m3")):
            both("layer", M, N, dtype, fmt, 81, ld=N + 3, shift=1)
        x, dy, gamma, beta = inputs(M, N, "bf16", 82)
        mean, rstd = f32(M), f32(M)
        fo.norm_forward("layer", x.t, gamma, beta, Mat(M, N, "bf16").t, M, N, "bf16", 1e-6, mean, rstd)
        work = torch.empty(fo.norm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
        for with_dx, with_g, with_b in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 0, 1)):
            dx, dg, db = Mat(M, N, "bf16") if with_dx else None, f32(N) if with_g else None, f32(N) if with_b else None
            fo.norm_backward("layer", dy.t, x.t, gamma, mean, rstd, dx.t if dx else None, dg, db, M, N, "bf16", work)
            torch.cuda.synchronize()
            check_backward("layer", "none", x, dy, gamma, mean, rstd, dx, dg, db, f"wide {M}x{N} {with_dx}{with_g}{with_b}")


def test_no_rows():
    torch = torch_mod()
    dg, db = f32(100, 5.0), f32(100, 5.0)
    fo.norm_backward("layer", None, None, None, None, None, None, dg, db, 0, 100, "bf16")
    torch.cuda.synchronize()
    assert (host(dg) == 0).all() and (host(db) == 0).all()


def test_extreme_rows():
    """Constant rows, rows of zeros, a mean far from zero, the type's largest values, infinities and NaN."""
    torch = torch_mod()
    N = 264
    rng = np.random.default_rng(41)
    for dtype, far, top in (("fp16", 1000.0, 65504.0), ("bf16", 300.0, 2.0 ** 60)):
        rows = [np.zeros(N), np.full(N, 3.0), far + rng.normal(size=N) * 4, np.where(rng.random(N) < 0.5, -top, top),
                rng.normal(size=N) * 2.0 ** -14]
        values = torch.as_tensor(np.stack(rows))
        given = (Mat(5, N, dtype, values=values), Mat(5, N, dtype, values=torch.as_tensor(rng.normal(size=(5, N)))),
                 vec(rng.uniform(0.5, 1.5, N), dtype), vec(rng.normal(size=N), dtype))
        for kind, fmt in itertools.product(["layer", "rms"], ["none", "int8", "e4m3"]):
            # (largest values of 2^60: the mean square, 2^120, stays in fp32's range)
            both(kind, 5, N, dtype, fmt, 0, given=given, eps=1e-5)
        bad = values.clone()
        bad[1, 7], bad[3, 200] = float("nan"), float("inf")
        x, y, mean, rstd = Mat(5, N, dtype, values=bad), Mat(5, N, dtype), f32(5), f32(5)
        codes, scales = kept_of(5, N)
        fo.norm_forward("layer", x.t, None, None, y.t, 5, N, dtype, 1e-5, mean, rstd, codes, scales)
        dx = Mat(5, N, dtype)
        fo.norm_backward("layer", given[1].t, None, None, mean, rstd, dx.t, None, None, 5, N, dtype, packed=codes, scales=scales)
        torch.cuda.synchronize()
        spoiled = np.array([False, True, False, True, False])
        np.testing.assert_array_equal(np.isnan(y.values()).all(axis=1), spoiled)
        np.testing.assert_array_equal(np.isnan(y.values()).any(axis=1), spoiled)
        np.testing.assert_array_equal(np.isnan(dx.values()).all(axis=1), spoiled)
        np.testing.assert_array_equal(np.isnan(dx.values()).any(axis=1), spoiled)


def test_gradient_against_differences():
    """The kernels' own forward pass in steps around x, gamma and beta (fp16 inputs on a grid that a step stays on)."""
    torch = torch_mod()
    M, N, dtype, d = 2, 24, "fp16", 2.0 ** -5
    rng = np.random.default_rng(51)
    grid = lambda *s: np.rint(rng.uniform(-2, 2, s) * 32) / 32
    x, dy, gamma, beta = grid(M, N), grid(M, N), grid(N) + 2.5, grid(N)

    def loss(x, gamma, beta):
        """<dy, y>, y in 64 bits from the statistics that the kernel computes (y itself has 11 bits only)."""
        m = Mat(M, N, dtype, values=torch.as_tensor(x))
        mean, rstd, y = f32(M), f32(M), Mat(M, N, dtype)
        fo.norm_forward("layer", m.t, vec(gamma, dtype), vec(beta, dtype), y.t, M, N, dtype, 1e-3, mean, rstd)
        torch.cuda.synchronize()
        h = (x - host(mean)[:, None]) * host(rstd)[:, None]
        np.testing.assert_allclose(y.values(), h * gamma + beta, rtol=2.0 ** -9, atol=2.0 ** -9)
        return (dy * (h * gamma + beta)).sum()
    mean, rstd, dx, dg, db = f32(M), f32(M), Mat(M, N, dtype), f32(N), f32(N)
    mx, md, g = Mat(M, N, dtype, values=torch.as_tensor(x)), Mat(M, N, dtype, values=torch.as_tensor(dy)), vec(gamma, dtype)
    fo.norm_forward("layer", mx.t, g, vec(beta, dtype), Mat(M, N, dtype).t, M, N, dtype, 1e-3, mean, rstd)
    work = torch.empty(fo.norm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
    fo.norm_backward("layer", md.t, mx.t, g, mean, rstd, dx.t, dg, db, M, N, dtype, work)
    torch.cuda.synchronize()
    for which, grad in ((0, dx.values()), (1, host(dg)), (2, host(db))):
        for i in list(np.ndindex(grad.shape))[::5]:
            at = [x, gamma, beta]
            ends = []
            for sign in (1, -1, 2, -2):
                v = [a.copy() for a in at]
                v[which][i] += sign * d
                ends.append(loss(*v))
            # fourth order in the step; what is left: d^4 / 30 of the fifth derivative (a few units here), the
            # statistics' 2^-23 over the step, and dx's own rounding
            slope = (8 * (ends[0] - ends[1]) - (ends[2] - ends[3])) / (12 * d)
            assert abs(slope - grad[i]) <= 2.0 ** -11 * abs(grad[i]) + 2e-3, (which, i, slope, grad[i])


def test_equal_calls_give_equal_bits_and_streams_differ():
    torch = torch_mod()
    M, N, dtype = 1500, 1032, "bf16"
    x, dy, gamma, beta = inputs(M, N, dtype, 61)
    got = []
    for stream in (None, torch.cuda.Stream(), torch.cuda.Stream()):
        torch.cuda.synchronize()
        y, dx, mean, rstd, dg, db = Mat(M, N, dtype), Mat(M, N, dtype), f32(M), f32(M), f32(N), f32(N)
        work = torch.empty(fo.norm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        fo.norm_forward("layer", x.t, gamma, beta, y.t, M, N, dtype, 1e-6, mean, rstd, stream=stream)
        fo.norm_backward("layer", dy.t, x.t, gamma, mean, rstd, dx.t, dg, db, M, N, dtype, work, stream=stream)
        torch.cuda.synchronize()
        got.append([y.bits(), dx.bits(), host(mean), host(rstd), host(dg), host(db)])
    for other in got[1:]:
        for a, b in zip(got[0], other):
            np.testing.assert_array_equal(a, b)


def test_refused_tensors():
    torch = torch_mod()
    x, dy, gamma, beta = inputs(4, 64, "bf16", 71)
    y = Mat(4, 64, "bf16")
    call = lambda x=x.t, gamma=gamma, y=y.t, dtype="bf16", **kw: fo.norm_forward("layer", x, gamma, None, y, 4, 64, dtype, **kw)
    call()
    for bad in (dict(x=x.t.float()), dict(x=x.t.half()), dict(dtype="fp16"), dict(x=x.t[:3]), dict(x=x.t.t().contiguous().t()),
                dict(x=x.t[:1].expand(4, 64)), dict(gamma=gamma.float()), dict(gamma=gamma[:63]), dict(mean=torch.zeros(3, device="cuda")),
                dict(rstd=torch.zeros(4, device="cuda", dtype=torch.int32)), dict(y=y.t.cpu()), dict(y=x.t[:, :64].reshape(-1)[1:]),
                dict(packed=torch.zeros(8, device="cuda", dtype=torch.uint8), scales=torch.zeros(8, device="cuda", dtype=torch.uint8)),
                dict(ldx=65)):
        with pytest.raises(ValueError):
            call(**bad)
    work = torch.empty(fo.norm_workspace_bytes(4, 64) - 1, dtype=torch.uint8, device="cuda")
    with pytest.raises(fo.FoError):
        fo.norm_backward("layer", dy.t, x.t, gamma, f32(4), f32(4), None, f32(64), None, 4, 64, "bf16", work)
    torch.cuda.synchronize()
