"""The row operators as a mixture-of-experts block uses them, around the framework's
own path: norm with an 8-bit checkpoint, tokens sorted by expert, the experts'
products (one weight, tiles of 64 rows) and their All-to-All through
fo.run_overlapped, rows combined with a second checkpoint, and the way back to the
gradient of the block's input. Each step is checked against the 64-bit reference
on the values that the step before it left on the GPU. The whole chain is then
captured into a graph and replayed on other inputs and other routings."""
import numpy as np
import pytest

import paper_2504_19519_amd as fo
from gpu_util import dev_plan, say, streams_apart, torch_mod
from oracle import rowops as ref
from rowops_util import F32, Mat, close, rounded
from test_gpu_norm import check_backward, check_forward, f32, host, kept_of, vec

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
    """Buffers and calls of one block: T tokens of H values, K of E experts each."""

    def __init__(self, T, K, E, H, dtype, fmt, seed):
        torch = torch_mod()
        self.T, self.K, self.E, self.H, self.dtype, self.fmt = T, K, E, H, dtype, fmt
        self.cap = -(-fo.route_capacity(T, K, E, 64) // 64) * 64
        mat = lambda M: Mat(M, H, dtype)
        self.x, self.y, self.out, self.dout, self.dy, self.dx = (mat(T) for _ in range(6))
        self.rows, self.prod, self.drows, self.dprod = (mat(self.cap) for _ in range(4))
        rng = np.random.default_rng(seed)
        self.W = Mat(H, H, dtype, values=torch.as_tensor(rng.normal(size=(H, H)) / np.sqrt(H)))
        self.Wt = Mat(H, H, dtype, values=self.W.t.t())
        self.gamma, self.beta = vec(rng.uniform(0.5, 1.5, H), dtype), vec(rng.normal(size=H), dtype)
        self.mean, self.rstd, self.dgamma, self.dbeta = f32(T), f32(T), f32(H), f32(H)
        self.kept_x, self.kept_rows = kept_of(T, H), kept_of(self.cap, H)
        i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
        self.ids, self.slot, self.pair = i32(T * K), i32(T * K), i32(self.cap)
        self.offsets, self.counts = i32(E + 1), i32(E)
        self.weights, self.dweights = f32(T * K), f32(T * K)
        self.norm_work = torch.empty(fo.norm_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
        self.sort_work = torch.empty(fo.route_workspace_bytes(T, K, E), dtype=torch.uint8, device="cuda")
        self.plan = fo.plan_groups(self.cap, H, H, dtype=dtype, tile_m=64, tile_n=64, pattern="rowmajor",
                                   sizes=[self.cap // 64 * (H // 64)], unit="tiles")
        self.rows.t.zero_(), self.drows.t.zero_()
        torch.cuda.synchronize()

    def draw(self, seed):
        torch = torch_mod()
        rng = np.random.default_rng(seed)
        self.x.t.copy_(torch.as_tensor(rng.normal(size=(self.T, self.H)) + rng.normal(size=(self.T, 1))))
        self.dout.t.copy_(torch.as_tensor(rng.normal(size=(self.T, self.H))))
        ids = np.minimum(rng.geometric(0.3, (self.T, self.K)) - 1, self.E - 1)
        ids[rng.random((self.T, self.K)) < 0.05] = -1
        self.ids.copy_(torch.as_tensor(ids.reshape(-1)))
        self.weights.copy_(torch.as_tensor(rng.uniform(0, 1, self.T * self.K)))
        torch.cuda.synchronize()

    def kept(self, which):
        return dict(packed=which[0], scales=which[1], fmt=self.fmt)

    def dispatch(self, stream=None):
        T, K, E, H, d = self.T, self.K, self.E, self.H, self.dtype
        fo.norm_forward("layer", self.x.t, self.gamma, self.beta, self.y.t, T, H, d, 1e-6, self.mean, self.rstd,
                        **self.kept(self.kept_x), stream=stream)
        fo.route_sort(self.ids, T, K, E, self.offsets, self.counts, self.slot, self.pair, self.sort_work, 64, stream=stream)
        fo.route_permute(self.y.t, self.slot, self.rows.t, T, K, H, d, self.cap, self.offsets, self.counts, E, stream=stream)

    def combine(self, stream=None):
        T, K, H, d = self.T, self.K, self.H, self.dtype
        fo.route_combine(self.prod.t, self.slot, self.weights, self.out.t, T, K, H, d, self.cap,
                         **self.kept(self.kept_rows), stream=stream)
        fo.route_combine_backward(self.dout.t, None, self.slot, self.weights, self.drows.t, self.dweights, T, K, H, d, self.cap,
                                  self.offsets, self.counts, self.E, **self.kept(self.kept_rows), stream=stream)

    def back(self, stream=None):
        T, K, H, d = self.T, self.K, self.H, self.dtype
        fo.route_combine(self.dprod.t, self.slot, None, self.dy.t, T, K, H, d, self.cap, stream=stream)
        fo.norm_backward("layer", self.dy.t, None, self.gamma, self.mean, self.rstd, self.dx.t, self.dgamma, self.dbeta, T, H, d,
                         self.norm_work, **self.kept(self.kept_x), stream=stream)

    def whole(self, stream=None):
        """Everything on one stream, the experts' products as plain GEMMs."""
        self.dispatch(stream)
        fo.gemm_signal_reorder(self.plan, None, self.rows.t, self.W.t, self.prod.t, None, stream)
        self.combine(stream)
        fo.gemm_signal_reorder(self.plan, None, self.drows.t, self.Wt.t, self.dprod.t, None, stream)
        self.back(stream)

    def results(self):
        torch = torch_mod()
        torch.cuda.synchronize()
        used = int(self.offsets[-1].item())
        mats = [m.t.view(torch.int16).clone() for m in (self.y, self.out, self.dy, self.dx)]
        mats += [m.t[:used].view(torch.int16).clone() for m in (self.rows, self.prod, self.drows, self.dprod)]
        return mats + [t.clone() for t in (self.mean, self.rstd, self.dgamma, self.dbeta, self.dweights, self.slot, self.counts,
                                           self.offsets, self.pair[:used], self.kept_x[0], self.kept_x[1])]


@pytest.mark.parametrize("dtype,fmt", [("bf16", "int8"), ("fp16", "e4m3")])
def test_block_around_the_all_to_all(dtype, fmt):
    torch = torch_mod()
    T, K, E, H, dests = 96, 2, 6, 256, 4
    say(f"[block] T={T} K={K} E={E} H={H} {dtype} {fmt}, All-to-All of {dests}")
    b = Block(T, K, E, H, dtype, fmt, 1)
    b.draw(2)
    b.dispatch()
    torch.cuda.synchronize()
    check_forward("layer", b.x, b.gamma, b.beta, b.y, b.mean, b.rstd, 1e-6, "norm")
    ids = b.ids.cpu().numpy().reshape(T, K)
    offsets, counts, slot, pair = ref.route_sort(ids, E, 64)
    np.testing.assert_array_equal(b.slot.cpu().numpy().reshape(T, K), slot)
    rows = b.rows.bits()
    np.testing.assert_array_equal(rows[np.flatnonzero(pair >= 0)], b.y.bits()[pair[pair >= 0] // K])
    assert (rows[:len(pair)][pair < 0] == 0).all()

    # the experts' products, each row sent back to the rank that its token came from
    token = np.where(pair >= 0, pair // K, 0)
    bucket = np.zeros(b.cap, np.int32)
    bucket[:len(token)] = token * dests // T
    tiles = b.cap // 64 * (H // 64)
    plan = fo.plan_groups(b.cap, H, H, dtype=dtype, tile_m=64, tile_n=64, pattern="subtoken", num_dest=dests, row_bucket=bucket,
                          sizes=[tiles // 2, tiles - tiles // 2], unit="tiles")
    table = dev_plan(plan)
    C, dst = (torch.empty(b.cap * H, dtype=torch.int16, device="cuda") for _ in range(2))
    counters = torch.zeros(plan.num_counters, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    s1, s2 = streams_apart()
    torch.cuda.synchronize()
    fo.run_overlapped(plan, table, b.rows.t, b.W.t, C, None, dst, b.prod.t, counters=counters, status_word=status,
                      gemm_stream=s1, comm_stream=s2)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    # a product of H terms in fp32, rounded once
    want = b.rows.values() @ b.W.values().T
    mag = np.abs(b.rows.values()) @ np.abs(b.W.values()).T
    close(b.prod.values(), want, rounded(want, dtype, H * F32 * mag), "products", dtype)

    b.combine()
    torch.cuda.synchronize()
    w = b.weights.cpu().numpy().reshape(T, K)
    want, mag = ref.combine(b.prod.values(), slot, w)
    close(b.out.values(), want, rounded(want, dtype, (K + 1) * F32 * mag), "combined", dtype)
    seen = ref.unpack(*ref.pack(b.prod.values(), fmt, dtype), H, fmt)
    grads, dw, dmag = ref.combine_grad(b.dout.values(), seen, slot, w, b.cap)
    close(host(b.dweights).reshape(T, K), dw, (H / 64 + 24) * F32 * dmag, "dweights")
    drows = b.drows.values()
    for r, g in grads.items():
        close(drows[r], g, rounded(g, dtype, F32 * np.abs(g)), "drows", dtype)
    assert (b.drows.bits()[:len(pair)][pair < 0] == 0).all()

    fo.gemm_signal_reorder(b.plan, None, b.drows.t, b.Wt.t, b.dprod.t, None)
    b.back()
    torch.cuda.synchronize()
    want, mag = ref.combine(b.dprod.values(), slot, None)
    close(b.dy.values(), want, rounded(want, dtype, (K + 1) * F32 * mag), "dy", dtype)
    check_backward("layer", fmt, b.x, b.dy, b.gamma, b.mean, b.rstd, b.dx, b.dgamma, b.dbeta, "norm backward")


@pytest.mark.parametrize("T,K,E,H,dtype,fmt", [(3, 2, 4, 128, "bf16", "int8"), (700, 4, 9, 192, "fp16", "e4m3"),
                                               (2500, 4, 16, 64, "bf16", "e4m3")])
def test_captured_and_replayed(T, K, E, H, dtype, fmt):
    """The last size has a sort of several workgroups."""
    torch = torch_mod()
    say(f"[block] graph T={T} K={K} E={E} H={H} {dtype} {fmt}")
    b, eager = Block(T, K, E, H, dtype, fmt, 3), Block(T, K, E, H, dtype, fmt, 3)
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
        b.drows.t.zero_(), eager.drows.t.zero_()
        b.rows.t.zero_(), eager.rows.t.zero_()
        for t in (b.dx, b.dy, b.out, b.y):
            t.t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager.whole()
        for k, (p, q) in enumerate(zip(b.results(), eager.results())):
            assert torch.equal(p, q), (seed, k)


def test_two_blocks_at_once():
    """Two blocks with buffers of their own on two streams, and one after the other."""
    torch = torch_mod()
    shapes = [(1500, 4, 12, 128, "bf16", "int8"), (900, 2, 5, 320, "bf16", "e4m3")]
    alone = [Block(*s, 8) for s in shapes]
    both = [Block(*s, 8) for s in shapes]
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
