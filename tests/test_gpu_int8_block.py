"""The 8-bit operators as a mixture-of-experts block uses them: the residual's norm into
8 bits, a projection of it, the experts' two products over the tokens that fo.route_sort
has put in order, rows put into 8 bits between them, the rows combined, and the norm's
backward pass. Each step is checked against the 64-bit reference on the values that the
step before it left on the GPU; the chain is then captured, replayed on other inputs and
other routings, and run beside another one."""
import numpy as np
import pytest

import paper_2504_19519_amd as fo
from gpu_util import say, torch_mod
from int8_util import (Codes, check_grads, check_norm_codes, check_quantized, f32_vec, kept_sum, product_bound, to_dtype)
from oracle import int8ops as ref
from oracle import rowops as rowref
from rowops_util import F32, Mat, close, rounded, torch_dtype

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = torch_mod()
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    fo.lib()
    yield
    torch.cuda.synchronize()


class Block:
    """Buffers and calls of one block: T tokens of H values, K of E experts each, of F inner
    values; a projection to Q columns."""

    def __init__(self, T, K, E, H, F, Q, dtype, align, seed):
        torch = torch_mod()
        self.T, self.K, self.E, self.H, self.F, self.Q, self.dtype, self.align = T, K, E, H, F, Q, dtype, align
        self.cap = fo.route_capacity(T, K, E, align)
        rng = np.random.default_rng(seed)
        self.x, self.res, self.h, self.out, self.dy, self.dh, self.dx = (Mat(T, H, dtype) for _ in range(7))
        self.q, self.up, self.down = Mat(T, Q, dtype), Mat(self.cap, F, dtype), Mat(self.cap, H, dtype)
        self.y8, self.up8 = Codes(T, H), Codes(self.cap, F)
        self.sy, self.sup, self.rstd, self.dgamma = f32_vec(T), f32_vec(self.cap), f32_vec(T), f32_vec(H)

        def weight(rows, n):
            w, c, s = Mat(rows, n, dtype, values=torch.as_tensor(rng.normal(size=(rows, n)) / np.sqrt(n))), Codes(rows, n), f32_vec(rows)
            fo.quantize_rows(w.t, c.whole, s, rows, n, dtype)
            return c, s
        self.wq, self.w1, self.w2 = weight(Q, H), weight(E * F, H), weight(E * H, F)
        self.gamma = torch.as_tensor(rng.uniform(0.5, 1.5, H)).cuda().to(torch_dtype(dtype))
        self.b1 = torch.as_tensor(rng.normal(size=(E, F))).cuda().to(torch_dtype(dtype))
        i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
        self.ids, self.slot, self.pair, self.offsets, self.counts = i32(T * K), i32(T * K), i32(self.cap), i32(E + 1), i32(E)
        self.weights = f32_vec(T * K)
        u8 = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
        self.sort_work, self.norm_work = u8(fo.route_workspace_bytes(T, K, E)), u8(fo.norm_workspace_bytes(T, H))
        self.q_work = u8(fo.int8_workspace_bytes(T, Q, H))
        torch.cuda.synchronize()

    def draw(self, seed):
        torch = torch_mod()
        rng = np.random.default_rng(seed)
        for m in (self.x, self.res, self.dy, self.dh):
            m.t.copy_(torch.as_tensor(rng.normal(size=(self.T, self.H)) * rng.uniform(0.3, 3, (self.T, 1))))
        ids = np.minimum(rng.geometric(0.3, (self.T, self.K)) - 1, self.E - 1)
        ids[rng.random((self.T, self.K)) < 0.05] = -1
        self.ids.copy_(torch.as_tensor(ids.reshape(-1)))
        self.weights.copy_(torch.as_tensor(rng.uniform(0, 1, self.T * self.K)))
        torch.cuda.synchronize()

    def whole(self, stream=None):
        T, K, E, H, F, Q, d, cap = self.T, self.K, self.E, self.H, self.F, self.Q, self.dtype, self.cap
        fo.norm_add_forward(self.x.t, self.res.t, self.gamma, self.h.t, None, T, H, d, 1e-6, rstd=self.rstd, codes=self.y8.whole,
                            scales=self.sy, stream=stream)
        fo.int8_product(self.y8.whole, self.sy, self.wq[0].whole, self.wq[1], self.q.t, T, Q, H, d, workspace=self.q_work,
                        stream=stream)
        fo.route_sort(self.ids, T, K, E, self.offsets, self.counts, self.slot, self.pair, self.sort_work, self.align, stream=stream)
        fo.int8_experts(self.y8.whole, self.sy, self.w1[0].whole, self.w1[1], self.up.t, F, H, E, d, cap, self.offsets, self.counts,
                        T, pair_of=self.pair, choices=K, bias=self.b1, stream=stream)
        fo.quantize_rows(self.up.t, self.up8.whole, self.sup, cap, F, d, stream=stream)
        fo.int8_experts(self.up8.whole, self.sup, self.w2[0].whole, self.w2[1], self.down.t, H, F, E, d, cap, self.offsets,
                        self.counts, cap, stream=stream)
        fo.route_combine(self.down.t, self.slot, self.weights, self.out.t, T, K, H, d, cap, stream=stream)
        fo.norm_add_backward(self.dy.t, self.dh.t, self.h.t, self.gamma, self.rstd, self.dx.t, self.dgamma, T, H, d, self.norm_work,
                             stream=stream)

    def results(self):
        torch = torch_mod()
        torch.cuda.synchronize()
        rows = self.slot[self.slot >= 0].long()
        mats = [m.t.view(torch.int16).clone() for m in (self.h, self.q, self.out, self.dx)]
        mats += [m.t[rows].view(torch.int16).clone() for m in (self.up, self.down)]
        return mats + [t.clone() for t in (self.y8.t, self.sy, self.up8.t[rows], self.sup[rows], self.rstd, self.dgamma, self.slot,
                                           self.counts)]

    def check(self):
        torch = torch_mod()
        torch.cuda.synchronize()
        T, K, E, H, F, d = self.T, self.K, self.E, self.H, self.F, self.dtype
        vec = lambda t: t.float().cpu().numpy().astype(np.float64)
        h = kept_sum(self.x.values(), self.res.values(), d)
        np.testing.assert_array_equal(self.h.values(), h)
        gamma, rstd = vec(self.gamma), vec(self.rstd)
        check_norm_codes(self.y8.values(), vec(self.sy), h, gamma, ref.norm_add(h, gamma, 1e-6)[0], "norm")
        want, mag = ref.product(self.y8.values(), vec(self.sy), self.wq[0].values(), vec(self.wq[1]))
        close(self.q.values(), want, product_bound(want, mag, d), "projection", d)
        offsets, counts, slot, pair = rowref.route_sort(self.ids.cpu().numpy().reshape(T, K), E, self.align)
        np.testing.assert_array_equal(self.slot.cpu().numpy().reshape(T, K), slot)

        def experts(got, a, sa, w, n, k, pairs, bias):
            want = ref.experts(a, sa, w[0].values().reshape(E, n, k), vec(w[1]).reshape(E, n), offsets, counts, self.cap, pairs, K, bias)
            rows = list(want)
            v, mag = (np.array([want[r][i] for r in rows]) for i in (0, 1))
            close(got.values()[rows], v, product_bound(v, mag, d), "experts", d)
            assert got.guards_stand(rows)
            return rows
        whole = np.full(self.cap, -1, np.int64)
        whole[:len(pair)] = pair
        rows = experts(self.up, self.y8.values(), vec(self.sy), self.w1, F, H, whole, vec(self.b1))
        check_quantized(self.up8.values()[rows], vec(self.sup)[rows].astype(np.float32), self.up.values()[rows], "between")
        experts(self.down, self.up8.values(), vec(self.sup), self.w2, H, F, None, None)
        want, mag = rowref.combine(self.down.values(), slot, vec(self.weights).reshape(T, K))
        close(self.out.values(), want, rounded(want, d, (K + 1) * F32 * mag), "combined", d)
        check_grads(self.dx.values(), vec(self.dgamma), self.dy.values(), self.dh.values(), h, gamma, rstd, d, "backward")


@pytest.mark.parametrize("T,K,E,H,F,Q,dtype,align", [(96, 2, 6, 256, 192, 128, "bf16", 64), (1, 2, 8, 130, 70, 33, "fp16", 1),
                                                     (300, 4, 9, 200, 321, 515, "fp16", 16), (17, 8, 60, 515, 64, 40, "bf16", 1)])
def test_block(T, K, E, H, F, Q, dtype, align):
    say(f"[int8 block] T={T} K={K} E={E} H={H} F={F} Q={Q} {dtype} align={align}")
    b = Block(T, K, E, H, F, Q, dtype, align, 1)
    b.draw(2)
    b.whole()
    b.check()


@pytest.mark.parametrize("T,K,E,H,F,Q,dtype", [(3, 2, 4, 8200, 64, 48, "bf16"), (700, 4, 9, 192, 320, 300, "fp16"),
                                               (4096, 2, 4, 520, 64, 4096, "bf16")])
def test_captured_and_replayed(T, K, E, H, F, Q, dtype):
    """The first size has a product in parts of k, the last one 256 x 256 tiles."""
    torch = torch_mod()
    say(f"[int8 block] graph T={T} K={K} E={E} H={H} F={F} Q={Q} {dtype}")
    b, eager = (Block(T, K, E, H, F, Q, dtype, 1, 3) for _ in range(2))
    assert H < 8200 or fo.int8_workspace_bytes(T, Q, H) > 0
    stream = torch.cuda.Stream()
    b.draw(4)
    b.whole(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.whole(stream)
    for seed in (5, 6, 7):
        b.draw(seed)
        eager.draw(seed)
        for m in (b.h, b.q, b.out, b.dx, b.up, b.down):
            m.t.fill_(float("nan"))
        for m in (eager.up, eager.down):
            m.t.fill_(float("nan"))
        b.q_work.fill_(0x7F), b.norm_work.fill_(0x7F)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager.whole()
        for k, (p, q) in enumerate(zip(b.results(), eager.results())):
            assert torch.equal(p, q), (seed, k)


def test_two_blocks_at_once():
    """Two blocks with buffers of their own on two streams, and one after the other."""
    torch = torch_mod()
    shapes = [(1500, 4, 12, 128, 200, 300, "bf16", 1), (4, 2, 5, 8320, 64, 30, "fp16", 1)]
    alone, both = [Block(*s, 8) for s in shapes], [Block(*s, 8) for s in shapes]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for k, b in enumerate(alone + both):
        b.draw(9 + k % 2)
    for b in alone:
        b.whole()
        torch.cuda.synchronize()
    for _ in range(3):
        for b, s in zip(both, (s1, s2)):
            b.whole(s)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for k, (p, q) in enumerate(zip(a.results(), b.results())):
            assert torch.equal(p, q), k
