"""A block of the 8-bit operators whose products all go in 256 x 256 tiles, several to a workgroup
(tests/int8_forms.py), captured once and replayed on other inputs and other routings, so that a
replay's workgroups have other tiles of other experts than those that were captured."""
import numpy as np
import pytest

import int8_forms as forms
import paper_2504_19519_amd as fo
from gpu_util import say, torch_mod
from test_gpu_int8_block import Block

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = torch_mod()
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    fo.lib()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_captured_and_replayed(dtype):
    torch = torch_mod()
    T, K, E, H, F, Q = (forms.TILED_BLOCK[k] for k in "TKEHFQ")
    say(f"[int8 tiles] graph {forms.TILED_BLOCK} {dtype}")
    b, eager = (Block(T, K, E, H, F, Q, dtype, 1, 3) for _ in range(2))
    stream = torch.cuda.Stream()
    b.draw(4)
    b.whole(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.whole(stream)
    counts = []
    for seed in (5, 6, 7, 8):
        for block in (b, eager):
            block.draw(seed)
            if seed == 7:           # all tokens to two experts; the others have none
                block.ids.copy_(torch.arange(T * K, device="cuda") % 2 * (E - 1))
            if seed == 8:           # most choices dropped: fewer tiles than compute units
                block.ids[T // 4:] = -1
            for m in (block.h, block.q, block.out, block.dx, block.up, block.down):
                m.t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager.whole()
        for k, (p, q) in enumerate(zip(b.results(), eager.results())):
            assert torch.equal(p, q), (seed, k)
        # rows that are no expert's are left as they were
        free = torch.ones(b.cap, dtype=torch.bool, device="cuda")
        free[b.slot[b.slot >= 0].long()] = False
        assert bool(torch.isnan(b.up.t[free]).all()) and bool(torch.isnan(b.down.t[free]).all())
        counts.append(b.counts.tolist())
    assert len({tuple(c) for c in counts}) == 4 and counts[2][1] == 0 and sum(counts[3]) < T


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_results(dtype):
    T, K, E, H, F, Q = (forms.TILED_BLOCK[k] for k in "TKEHFQ")
    say(f"[int8 tiles] {forms.TILED_BLOCK} {dtype}")
    b = Block(T, K, E, H, F, Q, dtype, 1, 9)
    b.draw(10)
    b.whole()
    b.check()
    assert np.isfinite(b.out.values()).all()
