"""The 8-bit operators on matrices past 4 GiB, whose element offsets pass 32 bits: the first
and the last rows against the 64-bit reference."""
import numpy as np
import pytest

import paper_2504_19519_amd as fo
from gpu_util import say, torch_mod
from int8_util import RSTD, check_grads, check_quantized, product_bound
from oracle import int8ops as ref
from rowops_util import F32, close, rounded

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


def ends(t, n=2):
    return np.concatenate([t[:n].double().cpu().numpy(), t[-n:].double().cpu().numpy()])


def test_rows_past_4_gib():
    torch = torch_mod()
    M, N = 70001, 32768
    say(f"[large] quantize and norm {M}x{N} bf16")
    x = torch.ones(M, N, dtype=torch.bfloat16, device="cuda")
    for rows in (slice(0, 2), slice(M - 2, M)):
        x[rows] = torch.randn(2, N, device="cuda").bfloat16()
    codes, scales = torch.zeros(M, N, dtype=torch.int8, device="cuda"), torch.zeros(M, device="cuda")
    fo.quantize_rows(x, codes, scales, M, N, "bf16")
    check_quantized(ends(codes).astype(np.int8), ends(scales.view(-1, 1)).reshape(-1).astype(np.float32), ends(x), "quantize")
    assert bool((codes[2:-2] == 127).all())
    y, rstd = torch.zeros_like(x), torch.zeros(M, device="cuda")
    fo.norm_add_forward(x, None, None, None, y, M, N, "bf16", 0.0, rstd=rstd)
    r, want = ref.norm_add(ends(x), None, 0.0)
    close(ends(y), want, rounded(want, "bf16", np.abs(want) * (RSTD + 2 * F32)), "y", "bf16")
    assert bool((y[2:-2] == 1).all())
    # dy = h = 1 on the rows between: the gradient is dh's, each adds 1 to every column's sum
    dgamma, work = torch.empty(N, device="cuda"), torch.empty(fo.norm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
    r = ends(rstd.view(-1, 1)).reshape(-1)
    fo.norm_add_backward(x, x, x, None, rstd, y, dgamma, M, N, "bf16", work)
    check_grads(ends(y), None, ends(x), ends(x), ends(x), None, r, "bf16", "dx")
    close(dgamma.cpu().numpy(), M - 4 + ref.norm_add_grad(ends(x), None, ends(x), None, r)[1], (M + 64) * F32 * (M + 64), "dgamma")


@pytest.mark.parametrize("K", [64, 300])
def test_product_past_4_gib(K):
    torch = torch_mod()
    M, N = 70001, 32776
    say(f"[large] product {M}x{N}x{K}")
    a = torch.randint(-128, 128, (M, fo.int8_row_bytes(K)), dtype=torch.int8, device="cuda")
    b = torch.randint(-128, 128, (N, fo.int8_row_bytes(K)), dtype=torch.int8, device="cuda")
    a[:, K:] = 0
    b[:, K:] = 0
    sa, sb = torch.rand(M, device="cuda") / 64, torch.rand(N, device="cuda") / 64
    c = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    fo.int8_product(a, sa, b, sb, c, M, N, K, "bf16")
    want, mag = ref.product(ends(a, 70)[:, :K].astype(np.int8), ends(sa.view(-1, 1), 70).reshape(-1), b[:, :K].cpu().numpy(),
                            sb.cpu().numpy())
    close(ends(c, 70), want, product_bound(want, mag, "bf16"), "c", "bf16")
    assert not bool(torch.isnan(c[:, ::97]).any())


def test_experts_past_4_gib():
    torch = torch_mod()
    E, N, K, T, choices = 40, 2048, 65536, 12, 3
    say(f"[large] experts {E}x{N}x{K}")
    b = torch.randint(-128, 128, (E, N, K), dtype=torch.int8, device="cuda")
    a = torch.randint(-128, 128, (T, K), dtype=torch.int8, device="cuda")
    sa, sb = torch.rand(T, device="cuda") / 4096, torch.rand(E, N, device="cuda") / 64
    ids = torch.tensor([[0, E - 1, t % E] for t in range(T)], dtype=torch.int32, device="cuda")
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32, device="cuda")
    offsets, counts, slot, pair = i32(E + 1), i32(E), i32(T, choices), i32(T * choices)
    fo.route_sort(ids, T, choices, E, offsets, counts, slot, pair)
    c = torch.full((T * choices, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    fo.int8_experts(a, sa, b, sb, c, N, K, E, "bf16", T * choices, offsets, counts, T, pair_of=pair, choices=choices)
    for t, k in ((0, 0), (3, 1), (T - 1, 1), (7, 2)):
        e, r = int(ids[t, k]), int(slot[t, k])
        want, mag = ref.product(a[t:t + 1].cpu().numpy(), sa[t:t + 1].cpu().numpy(), b[e].cpu().numpy(), sb[e].cpu().numpy())
        close(c[r:r + 1].double().cpu().numpy(), want, product_bound(want, mag, "bf16"), f"token {t} expert {e}", "bf16")
    assert not bool(torch.isnan(c).any())
