"""The 8-bit operators' refusals and sizes, and their reference, without a GPU."""
import numpy as np
import pytest

import paper_2504_19519_amd as fo
from oracle import int8ops as ref

P = 1 << 24          # stands for device memory; no call below gets as far as using it
ARG, SHAPE, UNSUPPORTED = -1, -2, -3


def refused(status, f, *args, **kw):
    with pytest.raises(fo.FoError) as e:
        f(*args, **kw)
    assert e.value.status == status, e.value


def test_quantize_refusals():
    def call(x=P, codes=2 * P, scales=3 * P, M=4, N=70, dtype="bf16", **kw):
        fo.quantize_rows(x, codes, scales, M, N, dtype, **kw)
    for bad in (dict(x=None), dict(codes=None), dict(scales=None), dict(x=P + 1), dict(codes=2 * P + 8), dict(scales=3 * P + 2),
                dict(M=-1), dict(N=-1), dict(ldx=69), dict(ldc=64), dict(ldc=88), dict(codes=P + 64), dict(scales=P),
                dict(scales=2 * P + 16), dict(x=2 * P)):
        refused(ARG, call, **bad)
    refused(SHAPE, call, M=1 << 31, codes=1 << 60, scales=1 << 61)
    refused(SHAPE, call, N=(1 << 30) + 1, codes=1 << 60)
    with pytest.raises(ValueError):
        call(dtype="fp32")
    assert fo.lib().fo_quantize_rows(2, 4, 64, P, 64, 2 * P, 64, 3 * P, None) == ARG
    call(M=0, x=None, codes=None, scales=None)
    call(N=0, x=None, codes=None, scales=None)


def test_norm_add_forward_refusals():
    def call(x=P, residual=2 * P, gamma=None, h=3 * P, y=4 * P, M=4, N=70, dtype="bf16", eps=1e-6, **kw):
        fo.norm_add_forward(x, residual, gamma, h, y, M, N, dtype, eps, **kw)
    both = dict(codes=5 * P, scales=6 * P)
    for bad in (dict(x=None), dict(y=None), dict(x=P + 1), dict(residual=2 * P + 1), dict(h=3 * P + 1), dict(y=4 * P + 1),
                dict(gamma=3), dict(rstd=2), dict(M=-1), dict(N=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(ldx=69),
                dict(ldr=69), dict(ldh=69), dict(ldy=69), dict(codes=5 * P), dict(scales=6 * P), dict(both, codes=5 * P + 8),
                dict(both, scales=6 * P + 2), dict(both, ldc=64), dict(both, ldc=88), dict(both, codes=P), dict(both, codes=2 * P),
                dict(both, codes=3 * P + 16), dict(both, codes=4 * P + 256), dict(h=P + 2), dict(y=2 * P + 2), dict(h=4 * P),
                dict(h=P, y=P), dict(h=P, ldh=72), dict(y=2 * P, ldy=140)):
        refused(ARG, call, **bad)
    refused(UNSUPPORTED, call, N=32769)
    refused(SHAPE, call, M=1 << 31)
    refused(SHAPE, call, **dict(both, ldc=(1 << 22) + 16))
    call(M=0, x=None, residual=None, h=None, y=None)
    call(N=0, x=None, residual=None, h=None, y=None)


def test_norm_add_backward_refusals():
    need = fo.norm_workspace_bytes(4, 64)

    def call(dy=P, dh=2 * P, h=3 * P, gamma=None, rstd=4 * P, dx=5 * P, dgamma=6 * P, M=4, N=64, dtype="fp16",
             workspace=7 * P, **kw):
        fo.norm_add_backward(dy, dh, h, gamma, rstd, dx, dgamma, M, N, dtype, workspace, **kw)
    for bad in (dict(dy=None), dict(h=None), dict(rstd=None), dict(rstd=4 * P + 2), dict(dx=None, dgamma=None),
                dict(workspace=None), dict(workspace=7 * P + 4), dict(dgamma=6 * P + 2), dict(gamma=1), dict(dy=P + 1),
                dict(dx=P + 2), dict(dx=2 * P + 32), dict(dx=3 * P + 2), dict(dx=3 * P, lddx=66), dict(lddy=63), dict(lddh=63),
                dict(ldh=63), dict(lddx=63), dict(M=-1), dict(N=-1), dict(dgamma=None, N=20000, workspace=None)):
        refused(ARG, call, **bad)
    refused(UNSUPPORTED, call, N=32769)
    refused(SHAPE, call, M=1 << 31)
    L = fo.lib()
    args = [0, 4, 64, P, 64, None, 64, 2 * P, 64, None, 3 * P, 4 * P, 64, 5 * P, 6 * P, need - 1, None]
    assert L.fo_norm_add_backward(*args) == ARG and b"workspace" in L.fo_last_error()


def test_product_refusals():
    def call(a=P, a_scales=2 * P, b=3 * P, b_scales=4 * P, c=5 * P, M=4, N=8, K=70, dtype="bf16", **kw):
        fo.int8_product(a, a_scales, b, b_scales, c, M, N, K, dtype, workspace=9 * P, **kw)
    for bad in (dict(a=None), dict(a_scales=None), dict(b=None), dict(b_scales=None), dict(c=None), dict(a=P + 8), dict(b=3 * P + 4),
                dict(a_scales=2 * P + 2), dict(b_scales=4 * P + 1), dict(c=5 * P + 1), dict(bias=1), dict(M=-1), dict(N=-1),
                dict(K=-1), dict(lda=64), dict(ldb=64), dict(lda=88), dict(ldb=88), dict(ldc=7), dict(c=P), dict(c=P + 100),
                dict(c=3 * P), dict(c=6 * P, bias=6 * P)):
        refused(ARG, call, **bad)
    refused(UNSUPPORTED, call, K=131072)
    refused(SHAPE, call, M=1 << 31)
    refused(SHAPE, call, N=1 << 31)
    refused(SHAPE, call, lda=(1 << 22) + 16)
    refused(SHAPE, call, M=1 << 24, N=1 << 24, c=1 << 60, b=1 << 55)
    call(M=0, a=None, a_scales=None, c=None)
    call(N=0, b=None, b_scales=None, c=None)
    need = fo.int8_workspace_bytes(4, 8, 16384)
    assert need >= 2 * 4 * 8 * 4
    args = [0, 4, 8, 16384, P, 16384, 2 * P, 3 * P, 16384, 4 * P, None, 5 * P, 8]
    for bad in ([None, 1 << 40, None], [9 * P, need - 1, None], [9 * P + 8, need, None]):
        assert fo.lib().fo_int8_product(*args, *bad) == ARG and b"workspace" in fo.lib().fo_last_error()
    for bad in (-1, 0, 1 << 40):
        assert fo.int8_workspace_bytes(bad, 4, 4) == 0
    assert fo.int8_workspace_bytes(4, 4, 131072) == 0


def test_experts_refusals():
    def call(a=P, a_scales=2 * P, b=3 * P, b_scales=4 * P, c=5 * P, N=8, K=70, E=4, dtype="bf16", capacity=16, offsets=6 * P,
             counts=7 * P, rows=8, **kw):
        fo.int8_experts(a, a_scales, b, b_scales, c, N, K, E, dtype, capacity, offsets, counts, rows, **kw)
    for bad in (dict(a=None), dict(a_scales=None), dict(b=None), dict(b_scales=None), dict(c=None), dict(offsets=None),
                dict(counts=None), dict(a=P + 8), dict(b=3 * P + 4), dict(offsets=6 * P + 2), dict(counts=7 * P + 1), dict(E=0),
                dict(E=1025), dict(capacity=-1), dict(rows=-1), dict(N=-1), dict(K=-1), dict(lda=64), dict(ldb=64), dict(ldc=7),
                dict(pair_of=8 * P, choices=0), dict(pair_of=8 * P, choices=65), dict(pair_of=8 * P + 2), dict(bias=1), dict(c=P),
                dict(c=3 * P + 80 * 31)):
        refused(ARG, call, **bad)
    refused(UNSUPPORTED, call, K=131072)
    refused(SHAPE, call, rows=1 << 31, c=1 << 60)
    refused(SHAPE, call, N=1 << 29, ldc=1 << 29, c=1 << 60)
    refused(SHAPE, call, rows=1 << 26, pair_of=8 * P, c=1 << 60)
    refused(SHAPE, call, capacity=1 << 30, N=1 << 20, E=1, c=1 << 61)
    call(capacity=0, c=None, offsets=None)
    call(N=0, b=None, c=None)
    call(rows=0, a=None)


def test_tensors_on_the_host_are_refused():
    torch = pytest.importorskip("torch")
    codes = torch.zeros(4, 64, dtype=torch.int8)
    with pytest.raises(ValueError, match="GPU"):
        fo.quantize_rows(P, codes, P, 4, 64, "bf16")
    with pytest.raises(ValueError, match="GPU"):
        fo.int8_product(codes, P, codes, P, P, 4, 4, 64, "bf16")


def test_sizes():
    assert [fo.int8_row_bytes(n) for n in (0, 1, 15, 16, 17, 70)] == [0, 16, 16, 16, 32, 80]
    assert fo.int8_row_bytes(-1) == 0


# ---- the reference -------------------------------------------------------------

def test_reference_quantize():
    x = np.array([[0.0, 0.0, 0.0], [127.0, -0.5, 1.5], [127.0, 2.5, -1.5], [254.0, 3.0, -254.0], [1.0, np.inf, 2.0],
                  [np.nan, 0.0, 1.0], [-1e-40, 1e-40, 0.0]])
    codes, scales = ref.quantize(x)
    np.testing.assert_array_equal(codes, [[0, 0, 0], [127, 0, 2], [127, 2, -2], [127, 2, -127], [0, 0, 0], [0, 0, 0],
                                          [-127, 127, 0]])
    np.testing.assert_array_equal(scales[:4], [0, 1, 1, 2])
    assert np.isnan(scales[4:6]).all()
    rng = np.random.default_rng(0)
    x = rng.normal(size=(50, 40))
    codes, scales = ref.quantize(x)
    assert (np.abs(codes * scales[:, None] - x) <= scales[:, None] / 2 * (1 + 1e-12)).all()


@pytest.mark.parametrize("affine,beside", [(True, True), (False, True), (True, False)])
def test_reference_norm_gradient_against_differences(affine, beside):
    rng = np.random.default_rng(1)
    M, N, eps, d = 3, 9, 1e-3, 1e-5
    h, dy, dh = (rng.normal(size=(M, N)) for _ in range(3))
    gamma = rng.normal(size=N)

    def loss(h, gamma):
        return (ref.norm_add(h, gamma if affine else None, eps)[1] * dy).sum() + ((h * dh).sum() if beside else 0.0)
    dx, dgamma = ref.norm_add_grad(dy, dh if beside else None, h, gamma if affine else None, ref.norm_add(h, gamma, eps)[0])
    for which, grad in ((0, dx), (1, dgamma)) if affine else ((0, dx),):
        for i in np.ndindex(grad.shape):
            lo, hi = [h.copy(), gamma.copy()], [h.copy(), gamma.copy()]
            lo[which][i] -= d
            hi[which][i] += d
            assert abs((loss(*hi) - loss(*lo)) / (2 * d) - grad[i]) < 1e-6


def test_reference_products():
    rng = np.random.default_rng(2)
    a, b = rng.integers(-128, 128, (6, 10)).astype(np.int8), rng.integers(-128, 128, (3, 5, 10)).astype(np.int8)
    sa, sb, bias = rng.random(6), rng.random((3, 5)), rng.normal(size=(3, 5))
    c, _ = ref.product(a, sa, b[0], sb[0], bias[0])
    for i, j in np.ndindex(6, 5):
        assert abs(c[i, j] - (sum(int(x) * int(y) for x, y in zip(a[i], b[0, j])) * sa[i] * sb[0, j] + bias[0, j])) < 1e-9
    got = ref.experts(a, sa, b, sb, [0, 4, 4, 8], [2, 0, 3], 6, pair_of=[3, 11, -1, -1, 0, 12], choices=2, bias=bias)
    assert sorted(got) == [0, 1, 4]           # row 5: token 6 of 6
    for r, s, e in ((0, 1, 0), (1, 5, 0), (4, 0, 2)):
        np.testing.assert_allclose(got[r][0], ref.product(a[s:s + 1], sa[s:s + 1], b[e], sb[e], bias[e])[0][0])


def test_outputs_that_overlap_other_arguments():
    """A scale, a bias or a place that a call would overwrite while it reads it."""
    def norm(x=P, residual=2 * P, gamma=None, h=3 * P, y=4 * P, codes=5 * P, scales=6 * P, rstd=7 * P):
        fo.norm_add_forward(x, residual, gamma, h, y, 4, 70, "bf16", codes=codes, scales=scales, rstd=rstd)
    for bad in (dict(rstd=6 * P), dict(rstd=6 * P + 12), dict(scales=5 * P + 16), dict(rstd=5 * P), dict(scales=P), dict(scales=2 * P + 4),
                dict(rstd=3 * P), dict(rstd=4 * P + 8), dict(gamma=3 * P + 2), dict(gamma=4 * P), dict(gamma=6 * P), dict(gamma=5 * P)):
        refused(ARG, norm, **bad)

    M, N, K = 4, 40, 8192
    need = fo.int8_workspace_bytes(M, N, K)
    assert need > 0

    def product(a=P, a_scales=2 * P, b=3 * P, b_scales=4 * P, bias=5 * P, c=6 * P, workspace=7 * P):
        fo.int8_product(a, a_scales, b, b_scales, c, M, N, K, "fp16", bias=bias, workspace=workspace)
    for bad in (dict(c=2 * P), dict(c=4 * P + 16), dict(c=5 * P), dict(c=3 * P + 32), dict(c=7 * P), dict(c=7 * P + need - 2),
                dict(workspace=P), dict(workspace=2 * P), dict(workspace=3 * P + 16), dict(workspace=4 * P), dict(workspace=5 * P)):
        refused(ARG, product, **bad)

    E, cap, rows = 3, 12, 5

    def experts(a=P, a_scales=2 * P, b=3 * P, b_scales=4 * P, bias=5 * P, c=6 * P, offsets=7 * P, counts=8 * P, pair_of=9 * P):
        fo.int8_experts(a, a_scales, b, b_scales, c, N, 64, E, "fp16", cap, offsets, counts, rows, pair_of=pair_of, choices=2, bias=bias)
    for at in (dict(a=6 * P), dict(a_scales=6 * P + 4), dict(b=6 * P + 16), dict(b_scales=6 * P), dict(bias=6 * P), dict(offsets=6 * P),
               dict(counts=6 * P + 8), dict(pair_of=6 * P + 4)):
        refused(ARG, experts, **at)
