"""Shapes of tensor arguments of the row operators, without a GPU: stand-ins for tensors
on a device, as the binding's checks see them."""
import pytest

import paper_2504_19519_amd as fo

torch = pytest.importorskip("torch")


class OnDevice:
    """A tensor on the host that says it is on device 0."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0


def args():
    a = fo._Args("bf16", None)
    a.device = 0            # (as after a first tensor on the current device)
    return a


def bf16(*shape):
    return OnDevice(torch.zeros(*shape, dtype=torch.bfloat16))


def test_matrices_of_another_width_are_refused():
    M, N = 6, 64
    for shape in ((M, N + 8), (M, 2 * N), (M + 1, N + 8), (2, 3, N + 8), (N, M), (2 * M, N // 2 + 8), (N, 2, M)):
        with pytest.raises(ValueError, match="rows of 64"):
            args().rows(bf16(*shape), M, N, None, "x")
    for shape, ld in (((M, N), None), ((M + 3, N), None), ((2, 3, N), None), ((M, 4, 16), None), ((M * N,), None), ((M * N + 5,), None),
                      ((M, N + 8), N + 8), ((M * (N + 8),), N + 8), ((M, N, 1), None)):
        p, step = args().rows(bf16(*shape), M, N, ld, "x")
        assert p and step == (ld or N)
    padded = bf16(M, N + 8)
    assert args().rows(OnDevice(padded.t[:, :N]), M, N, None, "x")[1] == N + 8
    assert args().rows(bf16(2, 8, 32), 1, 512, None, "x")[1] == 512          # one row of the whole tensor
    # calls of no values read nothing
    args().rows(bf16(0, 5), 0, 7, None, "x")
    args().rows(bf16(4, 5), 4, 0, None, "x")


def test_routing_of_another_width_is_refused():
    T, K = 5, 2

    def i32(*shape):
        return OnDevice(torch.zeros(*shape, dtype=torch.int32))
    for shape in ((T, K + 1), (K, T + 1), (T, 1, K + 2)):
        with pytest.raises(ValueError, match="rows of 2"):
            args().flat(i32(*shape), T * K, "slot_of", "i32", K)
    for shape in ((T, K), (T * K,), (T * K + 3,), (2 * T, K), (T + 1, 1, K), (T * K, 1)):
        args().flat(i32(*shape), T * K, "slot_of", "i32", K)
    args().flat(i32(4, 3), 0, "slot_of", "i32", K)
    args().flat(i32(1, 9), 7, "counts", "i32")                # a vector

    def u8(*shape):
        return OnDevice(torch.zeros(*shape, dtype=torch.uint8))
    M, N = 6, 90                                                # rows of three blocks
    args().pack(u8(M, 96), u8(M, 3), M, N, "int8")
    args().pack(u8(M + 1, 3, 32), u8(M * 3 + 4), M, N, "int8")
    for packed, scales in ((u8(M, 128), u8(M, 3)), (u8(M, 96), u8(M, 4))):
        with pytest.raises(ValueError, match="rows of"):
            args().pack(packed, scales, M, N, "int8")
