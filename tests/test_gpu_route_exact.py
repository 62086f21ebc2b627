"""The gradients of the combine for rows of every number of lanes, from whole numbers:
rows up to 15 in magnitude (which a checkpoint keeps exactly), dout up to 3, weights powers of
two. Every product and sum is then exact in fp32 (a sum of H products is below 45 H < 2^24), so
that results have to be equal in whatever order a form adds."""
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


# 8, 16, 32 and 64 lanes to a row, full and ragged; up to 2048 pairs and past them, where rows of more than 512
# values have a workgroup or a wave
@pytest.mark.parametrize("H", [5, 64, 100, 128, 200, 256, 300, 320, 448, 500, 512, 520, 576, 700, 1024, 1500, 2880, 7168])
@pytest.mark.parametrize("T", [60, 1030])
def test_whole_numbers(H, T):
    torch = torch_mod()
    K, E = 3, 7
    gen = torch.Generator(device="cuda").manual_seed(H + T)

    def whole(most, *shape):
        return torch.randint(-most, most + 1, shape, generator=gen, device="cuda")
    i32 = lambda n: torch.full((n,), -7, dtype=torch.int32, device="cuda")
    ids = torch.randint(-1, E, (T, K), generator=gen, device="cuda", dtype=torch.int32)
    cap = fo.route_capacity(T, K, E, 8)
    offsets, counts, slot = i32(E + 1), i32(E), i32(T * K)
    work = torch.empty(fo.route_workspace_bytes(T, K, E), dtype=torch.uint8, device="cuda")
    fo.route_sort(ids, T, K, E, offsets, counts, slot, None, work, 8)
    torch.cuda.synchronize()
    at = slot.view(T, K).long()
    there = at >= 0
    for dtype, fmt in (("fp16", "none"), ("bf16", "int8"), ("fp16", "e4m3"), ("bf16", "none")):
        say(f"[route] whole numbers T={T} H={H} {dtype} {fmt}")
        d = torch_dtype(dtype)
        rows, dout = whole(15, cap, H).to(d), whole(3, T, H).to(d)
        w = torch.exp2(whole(2, T, K).float())
        kept = {}
        if fmt != "none":
            a, b = fo.packed_bytes(cap, H)
            kept = dict(packed=torch.empty(a, dtype=torch.uint8, device="cuda"),
                        scales=torch.empty(b, dtype=torch.uint8, device="cuda"), fmt=fmt)
        out, drows = torch.empty(T, H, dtype=d, device="cuda"), torch.full((cap, H), 9.0, dtype=d, device="cuda")
        dw = torch.full((T, K), float("nan"), device="cuda")
        fo.route_combine(rows, slot, w, out, T, K, H, dtype, cap, **kept)
        fo.route_combine_backward(dout, None if kept else rows, slot, w, drows, dw, T, K, H, dtype, cap, offsets, counts, E, **kept)
        torch.cuda.synchronize()
        seen = torch.where(there[:, :, None], rows.double()[at.clamp(min=0)], 0.0)
        # (a sum of three products of up to 60, in quarters: exact, and rounded once)
        assert torch.equal(out, (seen * w.double()[:, :, None]).sum(1).float().to(d))
        assert torch.equal(dw.double(), (seen * dout.double()[:, None, :]).sum(2))
        want = (dout.double()[:, None, :] * w.double()[:, :, None]).to(d)           # up to 12, in quarters: exact
        assert torch.equal(drows[at[there]], want[there])
