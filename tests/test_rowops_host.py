"""The row operators' refusals and sizes, and their reference, without a GPU."""
import ctypes
import itertools

import numpy as np
import pytest

import oracle
import paper_2504_19519_amd as fo
from oracle import rowops as ref

P = 1 << 20          # stands for device memory; no call below gets as far as using it


def refused(status, f, *args, **kw):
    with pytest.raises(fo.FoError) as e:
        f(*args, **kw)
    assert e.value.status == status, e.value


ARG, SHAPE, UNSUPPORTED = -1, -2, -3


def test_norm_forward_refusals():
    def call(kind="layer", x=P, gamma=None, beta=None, y=2 * P, M=4, N=64, dtype="bf16", eps=1e-6, **kw):
        fo.norm_forward(kind, x, gamma, beta, y, M, N, dtype, eps, **kw)
    for bad in (dict(x=None), dict(y=None), dict(x=P + 1), dict(y=P + 1), dict(M=-1), dict(N=-1), dict(eps=-1.0),
                dict(eps=float("nan")), dict(ldx=63), dict(ldy=63), dict(gamma=3), dict(beta=5), dict(mean=2), dict(rstd=6),
                dict(packed=4 * P), dict(scales=4 * P), dict(packed=4 * P + 8, scales=5 * P), dict(y=P + 2),
                dict(ldx=128, ldy=128, y=P + 2 * 63), dict(ldx=128, ldy=128, y=P + 2 * 65), dict(ldx=128, ldy=130, y=P),
                dict(x=P + 2 * 64, ldx=128, ldy=64, y=P)):
        refused(ARG, call, **bad)
    refused(UNSUPPORTED, call, N=32769)
    refused(SHAPE, call, M=1 << 40, y=1 << 60)
    for bad in (dict(kind="batch"), dict(dtype="fp32"), dict(packed=4 * P, scales=5 * P, fmt="int4")):
        with pytest.raises((ValueError, KeyError)):
            call(**bad)
    assert fo.lib().fo_norm_forward(2, 1, 4, 64, P, 64, None, None, 1e-6, 2 * P, 64, None, None, None, None, 0, None) == ARG
    assert fo.lib().fo_norm_forward(0, 2, 4, 64, P, 64, None, None, 1e-6, 2 * P, 64, None, None, None, None, 0, None) == ARG
    assert fo.lib().fo_norm_forward(0, 1, 4, 64, P, 64, None, None, 1e-6, 2 * P, 64, None, None, 4 * P, 5 * P, 2, None) == ARG
    call(M=0, x=None, y=None)
    call(N=0, x=None, y=None)


def test_norm_backward_refusals():
    need = fo.norm_workspace_bytes(4, 64)

    def call(kind="layer", dy=P, x=2 * P, gamma=None, mean=3 * P, rstd=4 * P, dx=5 * P, dgamma=6 * P, dbeta=None, M=4, N=64,
             dtype="fp16", workspace=7 * P, **kw):
        fo.norm_backward(kind, dy, x, gamma, mean, rstd, dx, dgamma, dbeta, M, N, dtype, workspace, **kw)
    for bad in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dx=None, dgamma=None),
                dict(packed=P, scales=P), dict(x=None, packed=P), dict(x=None, scales=P), dict(workspace=None),
                dict(workspace=7 * P + 4), dict(dgamma=6 * P + 2), dict(dbeta=1), dict(dx=P + 2), dict(dx=2 * P + 32),
                dict(lddx=10), dict(ldx=10), dict(lddy=10), dict(M=-1), dict(N=-1)):
        refused(ARG, call, **bad)
    refused(UNSUPPORTED, call, N=32769)
    L = fo.lib()
    args = [0, 0, 4, 64, P, 64, 2 * P, 64, None, None, 0, None, 3 * P, 4 * P, 5 * P, 64, 6 * P, None, 7 * P, need - 1, None]
    assert L.fo_norm_backward(*args) == ARG and b"workspace" in L.fo_last_error()


def test_pack_refusals():
    for f in (lambda x=P, packed=2 * P, scales=3 * P, M=4, N=64, fmt="int8", **kw:
              fo.pack_rows(x, packed, scales, M, N, "fp16", fmt, **kw),
              lambda x=P, packed=2 * P, scales=3 * P, M=4, N=64, fmt="int8", ldx=None:
              fo.unpack_rows(packed, scales, x, M, N, "fp16", fmt, ldx)):
        for bad in (dict(x=None), dict(packed=None), dict(scales=None), dict(x=P + 1), dict(packed=2 * P + 8), dict(ldx=63),
                    dict(M=-1), dict(N=-2)):
            refused(ARG, f, **bad)
        refused(SHAPE, f, M=1 << 30)
        with pytest.raises(ValueError):
            f(fmt="fp8")
        f(M=0, x=None, packed=None, scales=None)


def test_route_refusals():
    def sort(ids=P, T=4, K=2, E=8, offsets=P, counts=P, slot_of=P, pair_of=P, align=1, **kw):
        fo.route_sort(ids, T, K, E, offsets, counts, slot_of, pair_of, align=align, **kw)
    for bad in (dict(ids=None), dict(offsets=None), dict(counts=None), dict(slot_of=None), dict(K=0), dict(K=65), dict(E=0),
                dict(E=1025), dict(align=0), dict(T=-1), dict(ids=P + 2), dict(ids=P + 4, id_bytes=8), dict(id_bytes=2),
                dict(offsets=P + 1), dict(pair_of=P + 2), dict(capacity=7), dict(T=100000)):
        refused(ARG, sort, **bad)
    refused(SHAPE, sort, T=1 << 30, workspace=P)
    refused(SHAPE, sort, T=1 << 20, align=1 << 30, workspace=P)

    def permute(x=P, slot_of=P, rows=2 * P, T=4, K=2, H=64, capacity=8, **kw):
        fo.route_permute(x, slot_of, rows, T, K, H, "bf16", capacity, **kw)

    def combine(rows=P, slot_of=P, weights=None, out=2 * P, T=4, K=2, H=64, capacity=8, **kw):
        fo.route_combine(rows, slot_of, weights, out, T, K, H, "bf16", capacity, **kw)

    def back(dout=P, rows=2 * P, slot_of=P, weights=None, drows=4 * P, dweights=P, T=4, K=2, H=64, capacity=8, **kw):
        fo.route_combine_backward(dout, rows, slot_of, weights, drows, dweights, T, K, H, "bf16", capacity, **kw)
    for f in (permute, combine, back):
        for bad in (dict(slot_of=None), dict(slot_of=P + 2), dict(K=0), dict(K=65), dict(T=-1), dict(H=-1), dict(capacity=-1),
                    dict(ldr=63), dict(rows=P + 1)):
            refused(ARG, f, **bad)
        refused(SHAPE, f, T=1 << 31)
        refused(SHAPE, f, T=1 << 28)
    for f in (permute, back):
        for bad in (dict(offsets=P), dict(counts=P), dict(offsets=P, counts=P, E=0), dict(offsets=P, counts=P, E=1025),
                    dict(offsets=P + 2, counts=P, E=8)):
            refused(ARG, f, **bad)
    refused(ARG, permute, x=None)
    refused(ARG, permute, x=2 * P)
    refused(ARG, permute, x=2 * P + 2 * 7 * 64)
    refused(ARG, combine, out=P + 2 * 64)
    refused(ARG, back, dout=4 * P)
    refused(ARG, back, dout=4 * P, ldr=128, lddr=128, lddo=130)
    for bad in (dict(out=None), dict(weights=P + 2), dict(packed=P), dict(scales=P), dict(packed=P + 8, scales=P)):
        refused(ARG, combine, **bad)
    for bad in (dict(dout=None), dict(drows=None, dweights=None), dict(rows=None), dict(packed=P, scales=P),
                dict(rows=None, packed=P), dict(dweights=P + 2), dict(drows=2 * P + 2), dict(lddr=3), dict(lddo=3)):
        refused(ARG, back, **bad)
    permute(T=0), combine(T=0), back(T=0)


def test_tensors_on_the_host_are_refused():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        fo.norm_forward("layer", x, None, None, x, 4, 64, "bf16")
    with pytest.raises(ValueError, match="GPU"):
        fo.pack_rows(P, torch.zeros(4 * 64, dtype=torch.uint8), P, 4, 64, "bf16")


def test_sizes():
    for T, K, E, align in itertools.product((0, 1, 5, 4096), (1, 8), (1, 7, 1024), (1, 64)):
        assert fo.route_capacity(T, K, E, align) == T * K + min(E, T * K) * (align - 1)
    assert fo.route_capacity(-1, 1, 1, 1) == 0
    assert fo.packed_bytes(3, 33) == (3 * 64, 3 * 2) and fo.packed_bytes(0, 5) == (0, 0)
    assert fo.norm_workspace_bytes(0, 64) == 0 and fo.norm_workspace_bytes(64, 0) == 0
    assert fo.norm_workspace_bytes(1, 64) >= 2 * 64 * 4


# ---- the reference -------------------------------------------------------------

@pytest.mark.parametrize("kind,affine", itertools.product(["layer", "rms"], [False, True]))
def test_reference_norm_gradient_against_differences(kind, affine):
    rng = np.random.default_rng(5)
    M, N, eps, d = 3, 7, 1e-3, 1e-5
    x, dy = rng.normal(size=(M, N)) + 0.5, rng.normal(size=(M, N))
    gamma, beta = (rng.normal(size=N), rng.normal(size=N)) if affine else (np.ones(N), np.zeros(N))

    def loss(x, gamma, beta):
        return (ref.norm(x, *ref.norm_stats(x, kind, eps), gamma, beta) * dy).sum()
    grads = ref.norm_grad(dy, x, *ref.norm_stats(x, kind, eps), gamma, kind)
    for which, grad in enumerate(grads):
        at = [x, gamma, beta]
        for i in np.ndindex(grad.shape):
            lo, hi = [v.copy() for v in at], [v.copy() for v in at]
            lo[which][i] -= d
            hi[which][i] += d
            assert abs((loss(*hi) - loss(*lo)) / (2 * d) - grad[i]) < 1e-6


def test_reference_combine_gradient_against_differences():
    rng = np.random.default_rng(6)
    rows, w, dout = rng.normal(size=(5, 4)), rng.normal(size=(3, 2)), rng.normal(size=(3, 4))
    slot = np.array([[0, 3], [-1, 4], [1, -1]])

    def loss(rows, w):
        return (ref.combine(rows, slot, w)[0] * dout).sum()
    drows, dw, _ = ref.combine_grad(dout, rows, slot, w, 5)
    full = np.zeros((5, 4))
    for s, g in drows.items():
        full[s] = g
    for i in np.ndindex(rows.shape):
        hi, lo = rows.copy(), rows.copy()
        hi[i] += 1e-4
        lo[i] -= 1e-4
        assert abs((loss(hi, w) - loss(lo, w)) / 2e-4 - full[i]) < 1e-8
    for i in np.ndindex(w.shape):
        hi, lo = w.copy(), w.copy()
        hi[i] += 1e-4
        lo[i] -= 1e-4
        assert abs((loss(rows, hi) - loss(rows, lo)) / 2e-4 - dw[i]) < 1e-8


def test_reference_e4m3_is_the_nearest_value():
    every = ref._from_e4m3(np.arange(127, dtype=np.uint8))          # code 127 is a NaN
    assert every[126] == 448 and every[1] == 2.0 ** -9 and (np.diff(every) > 0).all()
    np.testing.assert_array_equal(ref._to_e4m3(every), np.arange(127))
    mid = (every[1:] + every[:-1]) / 2
    code = ref._to_e4m3(mid)
    np.testing.assert_array_equal(code, np.arange(126) + (np.arange(126) & 1))       # ties to even
    np.testing.assert_array_equal(ref._to_e4m3(np.nextafter(mid, 0)), np.arange(126))
    np.testing.assert_array_equal(ref._to_e4m3(np.nextafter(mid, 1e9)), np.arange(1, 127))
    np.testing.assert_array_equal(ref._to_e4m3(-every[1:]), np.arange(1, 127) + 128)


@pytest.mark.parametrize("dtype,fmt", itertools.product(["fp16", "bf16"], ["int8", "e4m3"]))
def test_reference_checkpoint_error(dtype, fmt):
    """Every value within the bounds that include/fo.h states, every finite bit pattern as a block's largest."""
    bits = np.arange(0x7C00 if dtype == "fp16" else 0x7F80, dtype=np.uint16)
    top = oracle.decode(bits, dtype)
    rng = np.random.default_rng(7)
    share = rng.uniform(-1, 1, (len(top), 32)) * np.exp2(-rng.integers(0, 12, (len(top), 32)))
    x = oracle.decode(oracle.encode(top[:, None] * share, dtype), dtype)
    x[:, 5] = -top
    x = np.clip(x, -top[:, None], top[:, None])
    codes, scales = ref.pack(x, fmt, dtype)
    assert scales.max() < 255 and scales.min() >= 1
    got = ref.unpack(codes, scales, 32, fmt)
    step = np.exp2(scales.astype(float) - 127)
    e = np.frexp(top)[1] - 1
    if fmt == "int8":
        np.testing.assert_array_equal(step[top > 0, 0], np.exp2(np.maximum(e[top > 0] - 6, -126.0)))
        bound = np.where(np.abs(x) > 127.5 * step, step, step / 2)
        assert dtype == "fp16" or (np.abs(x) <= 127.5 * step).all()
    else:
        bound = np.maximum(np.abs(x) * 2.0 ** -4, step * 2.0 ** -10)
    assert (np.abs(got - x) <= bound).all()
    assert np.abs(got).max() <= (65504 if dtype == "fp16" else oracle.decode(np.array([0x7F7F], np.uint16), "bf16")[0])
    assert not np.isfinite(ref.unpack(*ref.pack(np.array([[np.inf] + [1.0] * 32]), fmt, dtype), 33, fmt)[0, :32]).any()
