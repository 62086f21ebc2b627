"""Rows of one value through every kernel form of the norm."""
import pytest

import paper_2504_19519_amd as fo
from gpu_util import say, torch_mod
from rowops_util import torch_dtype

pytestmark = pytest.mark.gpu


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
