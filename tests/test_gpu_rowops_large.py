"""Row operators on matrices past 4 GiB, whose element offsets pass 32 bits: the first
and the last rows against the 64-bit reference, the ones between by their number."""
import numpy as np
import pytest

import paper_2504_19519_amd as fo
from gpu_util import say, torch_mod
from oracle import rowops as ref
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


def ends(t):
    return np.concatenate([t[:2].double().cpu().numpy(), t[-2:].double().cpu().numpy()])


def test_norm_past_4_gib():
    torch = torch_mod()
    M, N = 70001, 32768
    say(f"[large] norm {M}x{N} bf16, int8 checkpoint")
    x = torch.ones(M, N, dtype=torch.bfloat16, device="cuda")
    x[:, ::2] = -1                      # mean 0, variance 1
    for rows in (slice(0, 2), slice(M - 2, M)):
        x[rows] = torch.randn(2, N, device="cuda").bfloat16()
    a, b = fo.packed_bytes(M, N)
    codes, scales = torch.empty(a, dtype=torch.uint8, device="cuda"), torch.empty(b, dtype=torch.uint8, device="cuda")
    y, mean, rstd = torch.zeros_like(x), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    fo.norm_forward("layer", x, None, None, y, M, N, "bf16", 0.0, mean, rstd, codes, scales, "int8")
    torch.cuda.synchronize()
    v = ends(x)
    m, r = ref.norm_stats(v, "layer", 0.0)
    want = ref.norm(v, m, r, None, None)
    close(ends(y), want, rounded(want, "bf16", 2.0 ** -16 * (np.abs(want) + 1)), "y")
    assert torch.equal(y[2:-2], x[2:-2]) and not bool(mean[2:-2].any())
    dx, dgamma = y, torch.empty(N, device="cuda")        # dy = x: g = h on the rows between, so their dx is 0
    work = torch.empty(fo.norm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
    fo.norm_backward("layer", x, None, None, mean, rstd, dx, dgamma, None, M, N, "bf16", work, packed=codes, scales=scales)
    torch.cuda.synchronize()
    seen = ref.unpack(*ref.pack(v, "int8", "bf16"), N, "int8")
    want, dg, _ = ref.norm_grad(v, seen, ends(mean.reshape(-1, 1)).reshape(-1), ends(rstd.reshape(-1, 1)).reshape(-1), None, "layer")
    # (the two means are of values around 1: 2^-17 of that, times h of up to 5 and rstd of about 1)
    close(ends(dx), want, rounded(want, "bf16", 2.0 ** -13), "dx")
    assert float(dx[2:-2].abs().max()) <= 2.0 ** -13
    # every row between adds 1 to every column
    close(dgamma.cpu().numpy(), dg + (M - 4), (M + 64) * F32 * (M + 64), "dgamma")


def test_route_past_4_gib():
    torch = torch_mod()
    T, K, E, H = 150001, 2, 16, 8192
    say(f"[large] route T={T} K={K} E={E} H={H} bf16, e4m3 checkpoint")
    ids = torch.stack([torch.arange(T, device="cuda") % E, torch.arange(T, device="cuda") // 7 % E], 1).int()
    cap = fo.route_capacity(T, K, E, 64)
    assert cap * H * 2 > 2 ** 32
    i32 = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")
    offsets, counts, slot, pair = i32(E + 1), i32(E), i32(T * K), i32(cap)
    work = torch.empty(fo.route_workspace_bytes(T, K, E), dtype=torch.uint8, device="cuda")
    fo.route_sort(ids, T, K, E, offsets, counts, slot, pair, work, 64)
    x = (torch.arange(T, device="cuda") % 256).bfloat16()[:, None].expand(T, H).contiguous()       # a token is known by its number
    x[:, 1] = (torch.arange(T, device="cuda") // 256 % 256).bfloat16()
    x[:, H - 1] = (torch.arange(T, device="cuda") // 65536).bfloat16()
    rows = torch.full((cap, H), 3.0, dtype=torch.bfloat16, device="cuda")
    fo.route_permute(x, slot, rows, T, K, H, "bf16", cap, offsets, counts, E)
    used = int(offsets[-1].item())
    known = rows[:used, [0, 1, H - 1]].float()
    token = torch.where(pair[:used] >= 0, pair[:used] // K, 0)
    want = torch.stack([token % 256, token // 256 % 256, token // 65536], 1).float() * (pair[:used] >= 0)[:, None]
    assert torch.equal(known, want) and bool((rows[used:] == 3).all())
    w = torch.full((T, K), 0.5, device="cuda")
    w[-1] = torch.tensor([0.25, 0.5], device="cuda")
    a, b = fo.packed_bytes(cap, H)
    codes, scales = torch.empty(a, dtype=torch.uint8, device="cuda"), torch.empty(b, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(x)
    fo.route_combine(rows, slot, w, out, T, K, H, "bf16", cap, codes, scales, "e4m3")
    torch.cuda.synchronize()
    assert torch.equal(out[:-1], x[:-1]) and torch.equal(out[-1].float(), x[-1].float() * 0.75)
    # one value in each of a few tokens' gradients, at the first and the last column
    at = torch.tensor([0, 1, 65537, T - 2, T - 1], device="cuda")
    dout = torch.zeros_like(x)
    dout[at, 0], dout[at, H - 1] = 1.0, 2.0
    drows, dw = rows, torch.full((T, K), 7.0, device="cuda")
    fo.route_combine_backward(dout, None, slot, w, drows, dw, T, K, H, "bf16", cap, offsets, counts, E, packed=codes, scales=scales,
                              fmt="e4m3")
    torch.cuda.synchronize()
    s = slot.reshape(T, K)[at].long()
    assert torch.equal(drows[s][:, :, 0].float(), w[at]) and torch.equal(drows[s][:, :, H - 1].float(), 2 * w[at])
    assert float(drows[:used].float().sum()) == float(w[at].sum()) * 3
    v = x[at].double().cpu().numpy()
    kept = ref.unpack(*ref.pack(v, "e4m3", "bf16"), H, "e4m3")
    np.testing.assert_array_equal(dw[at].double().cpu().numpy(), np.repeat((kept[:, 0] + 2 * kept[:, H - 1])[:, None], K, 1))
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert not bool(dw[rest].any())
