"""Tensors whose shape does not fit the call, on the GPU: a matrix of another width than
the call's rows is refused, and nothing is written; what holds whole rows is taken."""
import itertools

import pytest

import paper_2504_19519_amd as fo
from gpu_util import torch_mod

pytestmark = pytest.mark.gpu


def test_padded_matrices():
    """[M, N + 8] for rows of N: refused in each place, taken as a view or with its row distance."""
    torch = torch_mod()
    M, N, pad = 6, 64, 72
    wide = torch.randn(M, pad, device="cuda").bfloat16()
    x, y = wide[:, :N].contiguous(), torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    fo.norm_forward("layer", x, None, None, y, M, N, "bf16")
    for bad in (wide, wide.view(2, 3, pad), torch.cat([x, x]).t().contiguous()):
        with pytest.raises(ValueError, match="x: "):
            fo.norm_forward("layer", bad, None, None, y, M, N, "bf16")
    untouched = torch.full((M, pad), 3.0, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="y: "):
        fo.norm_forward("layer", x, None, None, untouched, M, N, "bf16")
    torch.cuda.synchronize()
    assert bool((untouched == 3).all())
    for good, kw in ((wide[:, :N], {}), (wide, dict(ldx=pad)), (wide.view(-1), dict(ldx=pad)), (x.view(2, 3, N), {}),
                     (x.view(M, 4, 16), {}), (x.view(-1), {}), (torch.cat([x, x]), {})):
        again = torch.zeros_like(y)
        fo.norm_forward("layer", good, None, None, again, M, N, "bf16", **kw)
        torch.cuda.synchronize()
        assert torch.equal(again, y)


def test_routing_of_another_width():
    """ids, slots and weights of [T, K + 1] for K choices, codes of another row length."""
    torch = torch_mod()
    T, K, E, H = 5, 2, 4, 96
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32, device="cuda")
    ids = torch.arange(T * K, device="cuda").remainder(E).int().view(T, K)
    offsets, counts, slot = i32(E + 1), i32(E), i32(T, K)
    fo.route_sort(ids, T, K, E, offsets, counts, slot)
    with pytest.raises(ValueError, match="ids: "):
        fo.route_sort(i32(T, K + 1), T, K, E, offsets, counts, slot)
    with pytest.raises(ValueError, match="slot_of: "):
        fo.route_sort(ids, T, K, E, offsets, counts, i32(T, K + 1))
    rows = torch.randn(T * K, H, device="cuda").bfloat16()
    w, out = torch.rand(T, K, device="cuda"), torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="weights: "):
        fo.route_combine(rows, slot, torch.rand(T, K + 1, device="cuda"), out, T, K, H, "bf16", T * K)
    u8 = lambda *n: torch.zeros(*n, dtype=torch.uint8, device="cuda")
    for packed, scales, what in ((u8(T * K, 128), u8(T * K, 3), "packed"), (u8(T * K, 96), u8(T * K, 4), "scales")):
        with pytest.raises(ValueError, match=what + ": "):
            fo.route_combine(rows, slot, w, out, T, K, H, "bf16", T * K, packed, scales)
    with pytest.raises(ValueError, match="dweights: "):
        fo.route_combine_backward(out, rows, slot, w, None, torch.empty(T, K + 1, device="cuda"), T, K, H, "bf16", T * K)
    # more rows of the right width, and flat buffers, are taken
    want = None
    for more in itertools.product((0, 1), repeat=2):
        s = torch.cat([slot, slot]) if more[0] else slot.view(-1)
        p, c = (u8(2 * T * K, 96), u8(2 * T * K, 3)) if more[1] else (u8(T * K * 96 + 5), u8(T * K, 3, 1))
        got = torch.zeros_like(out)
        fo.route_combine(rows, s, torch.cat([w, w]), got, T, K, H, "bf16", T * K, p, c)
        torch.cuda.synchronize()
        want = got if want is None else want
        assert torch.equal(got, want) and bool(want.any())
