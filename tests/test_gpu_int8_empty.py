"""Rows without values in 8 bits: the largest magnitude of nothing is 0, and so is the scale."""
import pytest

import paper_2504_19519_amd as fo
from gpu_util import torch_mod
from int8_util import f32_vec
from rowops_util import torch_dtype

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


@pytest.mark.parametrize("M", [1, 9, 70, 100001])
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_without_values_have_scale_zero(dtype, M):
    torch = torch_mod()
    s = f32_vec(M + 1)
    fo.quantize_rows(None, None, s, M, 0, dtype)
    assert not s[:M].any().item() and float(s[M]) == -7.0
    s = f32_vec(M + 1)
    fo.norm_add_forward(None, None, None, None, None, M, 0, dtype, codes=None, scales=s)
    assert not s[:M].any().item() and float(s[M]) == -7.0
    # tensors of that shape
    s = f32_vec(M)
    fo.quantize_rows(torch.empty(M, 0, dtype=torch_dtype(dtype), device="cuda"), torch.empty(M, 0, dtype=torch.int8, device="cuda"),
                     s, M, 0, dtype)
    assert not s.any().item()
