"""Every kernel form of the norm with all of its row groups at work over several rounds
of rows and a remainder, against the formulas in 64 bits (elementary torch operations
on the GPU), and rows of one value.

Inputs of the gradients are whole numbers (x up to 15 in magnitude, dy and gamma up to
3, means up to 3) and rstd a power of two, and a checkpoint keeps such x exactly: every
product and sum in fp32 is then exact below 2^24, so that dgamma and dbeta have to be
equal, whatever row a mistake would leave out. dx: the two sums are exact, the quotients
by N, their products and the two differences are off by 2^-24 each of what they are,
fewer than eight of them: 2^-21 of the sum of magnitudes. Forward: the bound of
test_gpu_norm."""
import pytest

import paper_2504_19519_amd as fo
from gpu_util import say, torch_mod
from rowops_util import HALF, TINY, torch_dtype

pytestmark = pytest.mark.gpu
S = 2.0 ** -18          # a row's sum against its magnitudes (test_gpu_norm)


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = torch_mod()
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    fo.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def f32(n):
    torch = torch_mod()
    return torch.full((n,), float("nan"), dtype=torch.float32, device="cuda")


def kept_of(M, N, fmt):
    torch = torch_mod()
    if fmt == "none":
        return {}
    a, b = fo.packed_bytes(M, N)
    return dict(packed=torch.full((a,), 77, dtype=torch.uint8, device="cuda"),
                scales=torch.full((b,), 77, dtype=torch.uint8, device="cuda"), fmt=fmt)


def within(got, want, bound, what):
    """Every value of `got`, none of them a NaN, within its bound."""
    err = (got.double() - want).abs() - bound
    assert bool((err <= 0).all()), f"{what}: {int((~(err <= 0)).sum())} of {err.numel()} outside, the farthest by {float(err.max())}"


def forward(kind, M, N, dtype, fmt, gen):
    torch = torch_mod()
    what = f"[forms] forward {kind} {M}x{N} {dtype} {fmt}"
    say(what)
    x = (torch.randn(M, N, generator=gen, device="cuda") + 3 * torch.randn(M, 1, generator=gen, device="cuda")).to(torch_dtype(dtype))
    gamma = (torch.rand(N, generator=gen, device="cuda") + 0.5).to(x.dtype)
    beta = torch.randn(N, generator=gen, device="cuda").to(x.dtype)
    y, mean, rstd, kept = torch.full_like(x, float("nan")), f32(M), f32(M), kept_of(M, N, fmt)
    fo.norm_forward(kind, x, gamma, beta, y, M, N, dtype, 1e-6, mean, rstd, **kept)
    torch.cuda.synchronize()
    for i in range(0, M, 4096):
        at = slice(i, i + 4096)
        v = x[at].double()
        mag = v.abs().mean(1)
        m = v.mean(1) if kind == "layer" else torch.zeros_like(mag)
        v -= m[:, None]
        r = 1 / torch.sqrt((v * v).mean(1) + 1e-6)
        h = v * r[:, None]
        within(mean[at], m, S * mag + 2.0 ** -24 * m.abs(), what + " mean")
        within(rstd[at], r, r * (2 * S + (S * mag * r) ** 2), what + " rstd")
        g, b = gamma.double(), beta.double()
        want = h * g + b
        off = S * (r * mag)[:, None] if kind == "layer" else 0.0
        extra = g.abs() * (h.abs() * 2 * S + off) + 2.0 ** -22 * ((g * h).abs() + b.abs())
        within(y[at], want, HALF[dtype] * (want.abs() + extra) + TINY[dtype] + extra, what + " y")
    if kept:        # the same checkpoint as pack_rows writes
        alone = kept_of(M, N, fmt)
        fo.pack_rows(x, alone["packed"], alone["scales"], M, N, dtype, fmt)
        torch.cuda.synchronize()
        assert torch.equal(kept["packed"], alone["packed"]) and torch.equal(kept["scales"], alone["scales"]), what


def backward(kind, M, N, dtype, fmt, gen):
    torch = torch_mod()
    what = f"[forms] backward {kind} {M}x{N} {dtype} {fmt}"
    say(what)

    def whole(most, *shape):
        return torch.randint(-most, most + 1, shape, generator=gen, device="cuda").to(torch_dtype(dtype))
    x, dy, gamma = whole(15, M, N), whole(3, M, N), whole(3, N)
    mean = whole(3, M).float() if kind == "layer" else None
    rstd = torch.exp2(torch.randint(-1, 2, (M,), generator=gen, device="cuda").float())
    kept = kept_of(M, N, fmt)
    if kept:
        fo.pack_rows(x, kept["packed"], kept["scales"], M, N, dtype, fmt)
    dx, dgamma, dbeta = torch.full_like(x, float("nan")), f32(N), f32(N)
    work = torch.full((fo.norm_workspace_bytes(M, N),), 0xFF, dtype=torch.uint8, device="cuda")
    fo.norm_backward(kind, dy, None if kept else x, gamma, mean, rstd, dx, dgamma, dbeta, M, N, dtype, work, **kept)
    torch.cuda.synchronize()
    dg, db = torch.zeros(N, dtype=torch.float64, device="cuda"), torch.zeros(N, dtype=torch.float64, device="cuda")
    most = torch.zeros_like(dg)
    for i in range(0, M, 4096):
        at = slice(i, i + 4096)
        r = rstd[at].double()[:, None]
        t = x[at].double() - (mean[at].double()[:, None] if mean is not None else 0)
        d = dy[at].double()
        dg, db, most = dg + (d * r * t).sum(0), db + d.sum(0), most + (d * r * t).abs().sum(0)
        g, h = d * gamma.double(), t * r
        a, b = (g.mean(1, keepdim=True) if mean is not None else torch.zeros_like(r)), (g * h).mean(1, keepdim=True)
        want = r * (g - a - h * b)
        extra = 2.0 ** -21 * r * (g.abs() + a.abs() + (h * b).abs())
        within(dx[at], want, HALF[dtype] * (want.abs() + extra) + TINY[dtype] + extra, what + " dx")
    # (halves of whole numbers: exact below 2^23)
    assert float(most.max()) < 2 ** 23
    assert torch.equal(dgamma.double(), dg), what + " dgamma"
    assert torch.equal(dbeta.double(), db), what + " dbeta"


# Columns of each class, and rows for each number of row groups that a class has, odd ones
# for a remainder; the last entry of a class has several rounds of rows per workgroup.
SIZES = [(40, 33001), (40, 70001), (100, 17003), (100, 33001), (128, 66001), (200, 8501), (200, 17001), (250, 34001),
         (400, 601), (400, 1101), (400, 2101), (500, 4101), (512, 17003),
         (800, 601), (800, 1101), (1000, 2101), (1024, 9001),
         (1600, 601), (1600, 1101), (2048, 2101), (1601, 5001),
         (3000, 771), (3000, 3001), (4096, 2051),
         (5000, 513), (8192, 771), (8191, 1033),
         (9001, 513), (12288, 771), (9001, 1033), (9001, 4099), (12288, 4097),
         (13000, 513), (16384, 771), (16383, 1033),
         (16391, 513), (20000, 771), (32767, 519), (32768, 773)]


@pytest.mark.parametrize("N,M", SIZES)
def test_rows_and_rounds(N, M):
    torch = torch_mod()
    gen = torch.Generator(device="cuda").manual_seed(M + N)
    for kind, dtype, fmt in (("layer", "bf16", "none"), ("layer", "fp16", "int8"), ("rms", "fp16", "e4m3"), ("rms", "bf16", "none"),
                             ("layer", "bf16", "e4m3")):
        forward(kind, M, N, dtype, fmt, gen)
        backward(kind, M, N, dtype, fmt, gen)


@pytest.mark.parametrize("N", [1, 3, 64, 100, 129, 300, 1000, 1023, 1032, 2047, 3001, 4104, 8191, 8203, 9001, 10240, 12287, 12288, 13000,
                               16383, 16384, 16391, 20001, 32761, 32767, 32768])
def test_rows_of_one_value(N):
    """The mean of a row of one value is that value and the row's result beta, with an eps far below the values'
    steps: differences from the mean of one fp32 step of 2^14 would come out as 0.89. (Sums within a wave, at most
    2055 values of 11 bits, are exact, and so is the difference of a wave's mean from the first wave's. rstd:
    eps rounded to fp32, and a root within 1.5 steps: below 2^-22.)"""
    torch = torch_mod()
    M = 1033
    for dtype, step in (("fp16", 16.0), ("bf16", 128.0)):
        say(f"[forms] one value per row {M}x{N} {dtype}")
        c = (1024 + torch.arange(M, device="cuda") % 1024).to(torch.float32) * 16 * (1 - 2.0 * (torch.arange(M, device="cuda") % 2))
        x = (c / step).round().mul(step).to(torch_dtype(dtype))[:, None].expand(M, N).contiguous()
        gamma = torch.ones(N, device="cuda").to(x.dtype)
        beta = torch.arange(N, device="cuda").remainder(17).to(x.dtype)
        for fmt in ("none", "int8"):
            y, mean, rstd = torch.full_like(x, float("nan")), f32(M), f32(M)
            fo.norm_forward("layer", x, gamma, beta, y, M, N, dtype, 1e-6, mean, rstd, **kept_of(M, N, fmt))
            torch.cuda.synchronize()
            assert torch.equal(mean, x[:, 0].float())
            assert torch.equal(y, beta.expand(M, N))
            within(rstd, torch.full((M,), 1e3, dtype=torch.float64, device="cuda"), 1e3 * 2.0 ** -22, "rstd")
