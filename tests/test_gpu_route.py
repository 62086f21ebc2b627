"""Tokens sorted by expert, permuted, combined, and the gradients, on the GPU
against the 64-bit reference.

Bounds: out is a sum of K products in fp32, (K + 1) * 2^-24 of the sum of
magnitudes, rounded once; drows one product, rounded to fp32 and then once more;
dweights a sum over H in which no chain has more than H / 64 + 24 additions."""
import itertools

import numpy as np
import pytest

import paper_2504_19519_amd as fo
from gpu_util import say, torch_mod
from oracle import rowops as ref
from rowops_util import F32, Mat, close, rounded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = torch_mod()
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    fo.lib()
    yield
    torch.cuda.synchronize()


def ints(n, fill=-7):
    torch = torch_mod()
    return torch.full((max(int(n), 1),), fill, dtype=torch.int32, device="cuda")


def device_sort(ids, E, align, id64=False, stream=None):
    torch = torch_mod()
    T, K = ids.shape
    d = torch.as_tensor(ids, dtype=torch.int64 if id64 else torch.int32).cuda()
    cap = fo.route_capacity(T, K, E, align)
    offsets, counts, slot, pair = ints(E + 1), ints(E), ints(T * K), ints(cap)
    work = torch.full((fo.route_workspace_bytes(T, K, E),), 0xFF, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    fo.route_sort(d, T, K, E, offsets, counts, slot, pair, work, align, stream=stream)
    torch.cuda.synchronize()
    return offsets, counts, slot, pair, cap


def check_sort(ids, E, align, id64=False):
    T, K = ids.shape
    say(f"[route] sort T={T} K={K} E={E} align={align} {'int64' if id64 else 'int32'}")
    offsets, counts, slot, pair, cap = device_sort(ids, E, align, id64)
    o, c, s, p = ref.route_sort(ids, E, align)
    np.testing.assert_array_equal(offsets.cpu().numpy()[:E + 1], o)
    np.testing.assert_array_equal(counts.cpu().numpy()[:E], c)
    np.testing.assert_array_equal(slot.cpu().numpy()[:T * K], s.reshape(-1))
    got = pair.cpu().numpy()
    np.testing.assert_array_equal(got[:len(p)], p)
    assert (got[len(p):] == -7).all()          # rows behind the last expert's are left


@pytest.mark.parametrize("T,K,E,align", [(0, 2, 8, 4), (1, 1, 1, 1), (1, 8, 256, 64), (5, 2, 3, 7), (16, 8, 256, 1), (100, 64, 65, 16),
                                         (63, 1, 2, 1), (1000, 1, 1000, 1), (4097, 2, 1024, 3), (1024, 8, 128, 64), (1025, 8, 60, 256),
                                         (2049, 4, 17, 128), (8192, 1, 1, 5), (9000, 3, 1024, 1), (40000, 2, 8, 64)])
def test_sort(T, K, E, align):
    rng = np.random.default_rng(T + K)
    check_sort(rng.integers(0, E, (T, K)), E, align)
    check_sort(rng.integers(-2, E + 2, (T, K)), E, align, True)              # dropped choices on both sides
    check_sort(np.minimum(rng.geometric(0.3, (T, K)) - 1, E - 1), E, align)  # uneven


def test_sort_borders():
    for E in (1, 2, 63, 64, 65, 1024):
        check_sort(np.full((300, 3), E - 1), E, 64)
        check_sort(np.full((300, 3), -1), E, 64)                            # nobody stays
        check_sort(np.arange(20000).reshape(-1, 2) % E, E, 2)
    big = np.full((40, 2), 5, np.int64)
    big[3], big[5], big[7] = 2 ** 32 + 5, -2 ** 40, 2 ** 31
    check_sort(big, 8, 1, True)                                             # ids past 32 bits are dropped, not cut off


def test_sort_million_pairs():
    """More pairs than 256 workgroups of one run: longer runs, against a stable argsort."""
    torch = torch_mod()
    T, K, E, align = 500000, 5, 100, 16
    say("[route] sort of 2.5 million pairs")
    ids = torch.randint(-1, E, (T, K), device="cuda", dtype=torch.int32)
    cap = fo.route_capacity(T, K, E, align)
    offsets, counts, slot, pair = ints(E + 1), ints(E), ints(T * K), ints(cap)
    work = torch.empty(fo.route_workspace_bytes(T, K, E), dtype=torch.uint8, device="cuda")
    fo.route_sort(ids, T, K, E, offsets, counts, slot, pair, work, align)
    torch.cuda.synchronize()
    flat = ids.cpu().numpy().reshape(-1)
    key = np.where(flat < 0, E, flat)
    c = np.bincount(key, minlength=E + 1)[:E]
    o = np.concatenate([[0], np.cumsum(-(-c // align) * align)])
    np.testing.assert_array_equal(counts.cpu().numpy(), c)
    np.testing.assert_array_equal(offsets.cpu().numpy(), o)
    order = np.argsort(key, kind="stable")[:c.sum()]
    want = np.full(len(flat), -1)
    start = np.concatenate([[0], np.cumsum(c)])[:E]
    want[order] = o[key[order]] + np.arange(len(order)) - start[key[order]]
    np.testing.assert_array_equal(slot.cpu().numpy(), want)


def whole(T, K, E, H, align, dtype, fmt, seed, ldx=None, ldr=None, shift=0, drop=0.1, weighted=True):
    """Every operator of one block on one routing."""
    torch = torch_mod()
    what = f"[route] T={T} K={K} E={E} H={H} align={align} {dtype} {fmt} ldx={ldx} ldr={ldr} shift={shift} weights={weighted}"
    say(what)
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, E, (T, K))
    ids[rng.random((T, K)) < drop] = -1
    if T > 2:
        ids[1] = -1                                  # a token that keeps no choice
    offsets, counts, slot, pair, cap = device_sort(ids, E, align)
    o, c, s, p = ref.route_sort(ids, E, align)
    filled, padding = np.flatnonzero(p >= 0), np.flatnonzero(p < 0)
    used = len(p)

    # permute
    x = Mat(T, H, dtype, ldx, shift, torch.as_tensor(rng.normal(size=(T, H))))
    rows = Mat(cap, H, dtype, ldr, shift)
    fo.route_permute(x.t, slot, rows.t, T, K, H, dtype, cap, offsets, counts, E)
    torch.cuda.synchronize()
    got = rows.bits()
    np.testing.assert_array_equal(got[filled], x.bits()[p[filled] // K], err_msg=what)
    assert (got[padding] == 0).all() and rows.guards_stand(range(used)), what
    bare = Mat(cap, H, dtype, ldr, shift)
    fo.route_permute(x.t, slot, bare.t, T, K, H, dtype, cap)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(bare.bits()[filled], got[filled])
    assert bare.guards_stand(filled), what

    # combine, with a checkpoint of the rows
    values = rng.normal(size=(cap, H)) * np.exp(rng.normal(size=(cap, 1)))
    values[padding] = np.nan                         # nothing is read there
    values[used:] = np.nan
    rows = Mat(cap, H, dtype, ldr, shift, torch.as_tensor(values))
    w = rng.uniform(-1, 1, (T, K)).astype(np.float32) if weighted else None
    if weighted:
        w[ids < 0] = np.nan                          # nor a dropped choice's weight used
    dw_in = torch.as_tensor(w).cuda() if weighted else None
    out = Mat(T, H, dtype, ldx, shift)
    kept = {}
    if fmt != "none":
        a, b = fo.packed_bytes(cap, H)
        kept = dict(packed=torch.full((a,), 99, dtype=torch.uint8, device="cuda"),
                    scales=torch.full((b,), 99, dtype=torch.uint8, device="cuda"), fmt=fmt)
    fo.route_combine(rows.t, slot, dw_in, out.t, T, K, H, dtype, cap, **kept)
    torch.cuda.synchronize()
    rv = rows.values()
    want, mag = ref.combine(rv, s, w)
    close(out.values(), want, rounded(want, dtype, (K + 1) * F32 * mag), what + " out", dtype)
    assert out.guards_stand(), what
    seen = rv
    if kept:
        with np.errstate(invalid="ignore"):
            codes, scales = ref.pack(rv, fmt, dtype)
        full_c, full_s = np.full_like(codes, 99), np.full_like(scales, 99)
        full_c[filled], full_s[filled] = codes[filled], scales[filled]
        np.testing.assert_array_equal(kept["scales"].cpu().numpy().reshape(full_s.shape), full_s, err_msg=what)
        np.testing.assert_array_equal(kept["packed"].cpu().numpy().reshape(full_c.shape), full_c, err_msg=what)
        seen = ref.unpack(codes, scales, H, fmt)

    # the gradients of the combine
    dout = Mat(T, H, dtype, ldx, shift, torch.as_tensor(rng.normal(size=(T, H))))
    drows = Mat(cap, H, dtype, ldr, shift)
    dweights = torch.full((T * K,), float("nan"), device="cuda")
    src = None if kept else rows.t
    fo.route_combine_backward(dout.t, src, slot, dw_in, drows.t, dweights, T, K, H, dtype, cap, offsets, counts, E, **kept)
    torch.cuda.synchronize()
    grads, dw, dmag = ref.combine_grad(dout.values(), seen, s, w, cap)
    got = drows.values()
    for r in filled:
        close(got[r], grads[int(r)], rounded(grads[int(r)], dtype, F32 * np.abs(grads[int(r)])), what + f" drows[{r}]", dtype)
    assert (drows.bits()[padding] == 0).all() and drows.guards_stand(range(used)), what
    close(dweights.cpu().numpy().reshape(T, K), dw, (H / 64 + 24) * F32 * dmag, what + " dweights")
    # one gradient alone, and drows over rows
    only = torch.full((T * K,), float("nan"), device="cuda")
    fo.route_combine_backward(dout.t, src, slot, dw_in, None, only, T, K, H, dtype, cap, **kept)
    alone = Mat(cap, H, dtype, ldr, shift)
    fo.route_combine_backward(dout.t, None, slot, dw_in, alone.t, None, T, K, H, dtype, cap)
    torch.cuda.synchronize()
    assert torch.equal(only, dweights), what
    np.testing.assert_array_equal(alone.bits()[filled], drows.bits()[filled])
    assert alone.guards_stand(filled), what
    if not kept:
        again = torch.full((T * K,), float("nan"), device="cuda")
        fo.route_combine_backward(dout.t, rows.t, slot, dw_in, rows.t, again, T, K, H, dtype, cap, offsets, counts, E)
        torch.cuda.synchronize()
        assert torch.equal(again, dweights), what
        np.testing.assert_array_equal(rows.bits()[:used], drows.bits()[:used])

    # the dispatch's backward pass: sums of the rows' gradient
    dx = Mat(T, H, dtype, ldx, shift)
    fo.route_combine(drows.t, slot, None, dx.t, T, K, H, dtype, cap)
    torch.cuda.synchronize()
    want, mag = ref.combine(drows.values(), s, None)
    close(dx.values(), want, rounded(want, dtype, (K + 1) * F32 * mag), what + " dx", dtype)


@pytest.mark.parametrize("H", [1, 7, 8, 9, 31, 32, 33, 100, 504, 511, 512, 513, 520, 1001, 2048, 2880, 7168])
def test_lengths(H):
    for i, (dtype, fmt) in enumerate(itertools.product(["fp16", "bf16"], ["none", "int8", "e4m3"])):
        whole(9, 3, 5, H, 4, dtype, fmt, H + i)


@pytest.mark.parametrize("H", [16, 56, 65, 72, 120, 128, 136, 200, 250, 256, 264, 300, 320, 448, 576, 700])
def test_lanes(H):
    """Slices of 8, 16, 32 and 64 lanes, full and ragged, few pairs and many."""
    whole(30, 2, 3, H, 1, "bf16", "none", H)
    whole(30, 2, 3, H, 8, "fp16", "e4m3", H + 1)
    if H in (72, 250, 576):
        whole(700, 3, 5, H, 4, "bf16", "int8", H + 2)
        whole(700, 3, 5, H, 1, "fp16", "none", H + 3)


@pytest.mark.parametrize("T,K,E,align", [(1, 1, 1, 1), (1, 8, 256, 1), (3, 1, 4, 64), (16, 2, 8, 64), (7, 64, 300, 1), (130, 5, 6, 16),
                                         (33, 9, 1024, 2), (257, 4, 3, 256), (12, 16, 16, 1), (20, 6, 60, 1)])
def test_routings(T, K, E, align):
    whole(T, K, E, 136, align, "bf16", "none", T)
    whole(T, K, E, 72, align, "fp16", "int8", T + 1, weighted=False)
    whole(T, K, E, 40, align, "fp16", "e4m3", T + 2, drop=0.9)


@pytest.mark.parametrize("H,ldx,ldr,shift", [(64, 64, 72, 1), (100, 103, 101, 3), (513, 1000, 514, 5), (1024, 1032, 2048, 8)])
def test_strides_and_alignment(H, ldx, ldr, shift):
    for fmt in ("none", "int8", "e4m3"):
        whole(11, 2, 4, H, 8, "bf16", fmt, 5, ldx, ldr, shift)


def test_one_token_beside_its_rows():
    """One token whose values lie between two of the rows that they go to."""
    torch = torch_mod()
    say("[route] one token beside its rows")
    H, K = 64, 2
    block = torch.zeros(K, 2 * H, dtype=torch.bfloat16, device="cuda")
    block[0, H:] = torch.arange(H, dtype=torch.bfloat16, device="cuda")
    x, rows = block[:1, H:], block[:, :H]
    slot = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    fo.route_permute(x, slot, rows, 1, K, H, "bf16", K)
    torch.cuda.synchronize()
    assert torch.equal(rows, x.expand(K, H))
    out = block[1:, H:]
    fo.route_combine(rows, slot, None, out, 1, K, H, "bf16", K)
    torch.cuda.synchronize()
    assert torch.equal(out, 2 * x)              # even integers up to 126: exact
    with pytest.raises(fo.FoError):
        fo.route_combine(rows, slot, None, block[:1, H - 1:2 * H - 1], 1, K, H, "bf16", K)


def test_slots_outside_the_rows_are_skipped():
    torch = torch_mod()
    T, K, H, cap = 4, 2, 64, 3
    slot = torch.tensor([[0, 3], [-5, 2], [2 ** 31 - 1, 1], [-2 ** 31, 7]], dtype=torch.int32, device="cuda")
    x = Mat(T, H, "fp16", values=torch.randn(T, H, dtype=torch.float64))
    rows, out, drows = Mat(cap, H, "fp16"), Mat(T, H, "fp16"), Mat(cap, H, "fp16")
    dw = torch.full((T * K,), 9.0, device="cuda")
    fo.route_permute(x.t, slot, rows.t, T, K, H, "fp16", cap)
    fo.route_combine(rows.t, slot, None, out.t, T, K, H, "fp16", cap)
    fo.route_combine_backward(x.t, rows.t, slot, None, drows.t, dw, T, K, H, "fp16", cap)
    torch.cuda.synchronize()
    v = x.bits()
    np.testing.assert_array_equal(rows.bits(), v[[0, 2, 1]])
    np.testing.assert_array_equal(out.values(), np.stack([x.values()[0], x.values()[1], x.values()[2], np.zeros(H)]))
    np.testing.assert_array_equal(drows.bits(), v[[0, 2, 1]])
    np.testing.assert_array_equal(dw.cpu().numpy() != 0, [True, False, False, True, False, True, False, False])
    assert rows.guards_stand() and drows.guards_stand() and out.guards_stand()
    # no rows at all
    fo.route_combine(None, slot, None, out.t, T, K, H, "fp16", 0)
    fo.route_combine_backward(x.t, None, slot, None, None, dw, T, K, H, "fp16", 0)
    torch.cuda.synchronize()
    assert (out.bits() == 0).all() and not bool(dw.any())


def test_spoiled_rows_stay_where_they_are():
    """An infinity or a NaN in one token's row reaches that token only."""
    torch = torch_mod()
    T, K, H = 6, 2, 128
    slot = torch.arange(T * K, dtype=torch.int32, device="cuda")
    values = torch.randn(T * K, H, dtype=torch.float64)
    values[4, 3], values[9, 100] = float("nan"), float("inf")
    rows, out = Mat(T * K, H, "bf16", values=values), Mat(T, H, "bf16")
    w = torch.ones(T, K, device="cuda")
    a, b = fo.packed_bytes(T * K, H)
    codes, scales = torch.zeros(a, dtype=torch.uint8, device="cuda"), torch.zeros(b, dtype=torch.uint8, device="cuda")
    fo.route_combine(rows.t, slot, w, out.t, T, K, H, "bf16", T * K, codes, scales, "e4m3")
    dw = torch.zeros(T * K, device="cuda")
    fo.route_combine_backward(out.t, None, slot, w, None, dw, T, K, H, "bf16", T * K, packed=codes, scales=scales, fmt="e4m3")
    torch.cuda.synchronize()
    bad = ~np.isfinite(out.values())
    assert bad.sum() == 2 and bad[2, 3] and bad[4, 100]
    np.testing.assert_array_equal(np.flatnonzero(~np.isfinite(dw.cpu().numpy())), [4, 5, 8, 9])


def test_streams_and_repeats():
    torch = torch_mod()
    rng = np.random.default_rng(3)
    ids = rng.integers(-1, 64, (5000, 6))
    first = device_sort(ids, 64, 64)
    for stream in (torch.cuda.Stream(), torch.cuda.Stream()):
        again = device_sort(ids, 64, 64, stream=stream)
        for a, b in zip(first[:4], again[:4]):
            assert torch.equal(a, b)


def test_refused_tensors():
    torch = torch_mod()
    slot, rows, x = ints(8, 0), Mat(8, 64, "bf16"), Mat(4, 64, "bf16")
    w = torch.zeros(4, 2, device="cuda")
    call = lambda slot=slot, rows=rows.t, w=w, out=x.t, **kw: fo.route_combine(rows, slot, w, out, 4, 2, 64, "bf16", 8, **kw)
    for bad in (dict(slot=slot.long()), dict(slot=slot[:7]), dict(rows=rows.t[:7]), dict(rows=rows.t.float()), dict(w=w.half()),
                dict(w=w.t()), dict(out=x.t[:3]), dict(out=x.t.cpu()), dict(slot=slot.float())):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(ValueError):
        fo.route_sort(ints(8), 4, 2, 8, ints(8), ints(8), ints(8))          # offsets: E + 1
    with pytest.raises(ValueError):
        fo.route_sort(torch.zeros(8, device="cuda"), 4, 2, 8, ints(9), ints(8), ints(8))
