"""The magnitudes that fo_norm_add_forward is described for, without an eps to help, at both
ends: rows of that size throughout and rows of one such value, forward and backward."""
import numpy as np
import pytest

import paper_2504_19519_amd as fo
from gpu_util import torch_mod
from int8_util import RSTD, Codes, F32, check_grads, check_norm_codes, f32_vec, to_dtype
from oracle import int8ops as ref
from rowops_util import Mat, close, rounded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = torch_mod()
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    fo.lib()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("N", [5, 8, 130, 3000, 16384, 32768])
@pytest.mark.parametrize("size", [2.0 ** -50, 2.0 ** -30, 2.0 ** 60])
def test_without_eps(size, N):
    torch = torch_mod()
    dtype, M = "bf16", 3
    rng = np.random.default_rng(N)
    hv = to_dtype(rng.uniform(0.5, 1.0, (M, N)) * rng.choice([-1, 1], (M, N)) * size, dtype)
    hv[1] = size
    hv[2] = 0.0
    hv[2, N // 2] = size
    mat = lambda v=None: Mat(M, N, dtype, values=None if v is None else torch.as_tensor(v))
    H, Y, C, s, rstd = mat(hv), mat(), Codes(M, N), f32_vec(M), f32_vec(M)
    fo.norm_add_forward(H.t, None, None, None, Y.t, M, N, dtype, 0.0, rstd=rstd, codes=C.whole, scales=s)
    want_r, want = ref.norm_add(hv, None, 0.0)
    close(rstd.cpu().numpy(), want_r, want_r * RSTD, "rstd")
    close(Y.values(), want, rounded(want, dtype, np.abs(want) * (RSTD + 2 * F32)), "y", dtype)
    check_norm_codes(C.values(), s.cpu().numpy(), hv, None, want_r, "codes")
    # (gradients of the gradients' usual size: dx is up to 1 / size of them)
    dyv = to_dtype(rng.normal(size=(M, N)), dtype)
    dx, dgamma = mat(), f32_vec(N)
    work = torch.full((fo.norm_workspace_bytes(M, N),), 0xFF, dtype=torch.uint8, device="cuda")
    fo.norm_add_backward(mat(dyv).t, None, H.t, None, rstd, dx.t, dgamma, M, N, dtype, work)
    check_grads(dx.values(), dgamma.cpu().numpy(), dyv, None, hv, None, rstd.cpu().numpy().astype(np.float64), dtype, "backward")
