"""Products over no inner values (K = 0): the bias, or zeros, whatever stands where the
scales are."""
import numpy as np
import pytest

import paper_2504_19519_amd as fo
from gpu_util import torch_mod
from int8_util import f32_vec, to_dtype
from rowops_util import GUARD, Mat, torch_dtype

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


SCALES = [float("nan"), float("inf"), -float("inf"), 0.0, 3.0e38]


# (of every form that K = 0 takes: few blocks, blocks of 32, 64 x 32, 64, 128 x 64, 128)
@pytest.mark.parametrize("M,N", [(2, 50), (30, 9000), (64, 5000), (64, 9000), (70, 9000), (300, 50), (1000, 5000)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_products_of_nothing_leave_the_scales_alone(dtype, M, N):
    torch = torch_mod()
    bias = to_dtype(np.random.default_rng(M).normal(size=N), dtype)
    sa = torch.tensor(SCALES, device="cuda").repeat(M // 5 + 1)[:M].contiguous()
    sb = torch.tensor(SCALES, device="cuda").repeat(N // 5 + 1)[:N].flip(0).contiguous()
    for b, want in ((bias, bias), (None, np.zeros(N))):
        C = Mat(M, N, dtype, N + 3)
        fo.int8_product(None, sa, None, sb, C.t, M, N, 0, dtype, bias=None if b is None else torch.as_tensor(b).cuda().to(torch_dtype(dtype)))
        assert fo.int8_workspace_bytes(M, N, 0) == 0
        np.testing.assert_array_equal(C.values(), np.broadcast_to(want, (M, N)))
        assert C.guards_stand()


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("counts,N", [([3, 0, 4], 33), ([300, 0, 70, 5], 70), ([2000, 0, 900], 700)])
def test_experts_products_of_nothing_leave_the_scales_alone(counts, N, gather):
    torch = torch_mod()
    dtype, E, gap = "bf16", len(counts), 2
    offsets = np.concatenate([[0], np.cumsum(np.array(counts) + gap)]).astype(np.int32)
    cap = int(offsets[-1])
    bias = to_dtype(np.random.default_rng(N).normal(size=(E, N)), dtype)
    dev = lambda v: torch.as_tensor(np.ascontiguousarray(v)).cuda()
    sa = torch.tensor(SCALES, device="cuda").repeat(cap // 5 + 1)[:cap].contiguous()
    sb = torch.tensor(SCALES, device="cuda").repeat(E * N // 5 + 1)[:E * N].reshape(E, N).contiguous()
    C = Mat(cap, N, dtype)
    fo.int8_experts(None, sa, None, sb, C.t, N, 0, E, dtype, cap, dev(offsets), dev(np.array(counts, np.int32)), cap,
                    pair_of=dev(np.arange(cap, dtype=np.int32)) if gather else None, bias=dev(bias).to(torch_dtype(dtype)))
    bits, got = C.raw.cpu().numpy()[:cap * N].reshape(cap, N), C.values()
    for e, n in enumerate(counts):
        np.testing.assert_array_equal(got[offsets[e]:offsets[e] + n], np.broadcast_to(bias[e], (n, N)))
        assert (bits[offsets[e] + n:offsets[e + 1]] == GUARD).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_from_rows_to_the_bias(dtype):
    """A layer of no inner values as it is used: its rows put into 8 bits, then the product. Memory that a
    program reuses holds anything, NaN too."""
    torch = torch_mod()
    M, N = 40, 60
    sa, sb = f32_vec(M, float("nan")), f32_vec(N, float("nan"))
    bias = to_dtype(np.random.default_rng(5).normal(size=N), dtype)
    fo.quantize_rows(None, None, sa, M, 0, dtype)
    fo.quantize_rows(None, None, sb, N, 0, dtype)
    C = Mat(M, N, dtype)
    fo.int8_product(None, sa, None, sb, C.t, M, N, 0, dtype, bias=torch.as_tensor(bias).cuda().to(torch_dtype(dtype)))
    np.testing.assert_array_equal(C.values(), np.broadcast_to(bias, (M, N)))
