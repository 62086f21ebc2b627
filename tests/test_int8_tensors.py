"""Shapes of tensors of codes, without a GPU: stand-ins for tensors on a device, as the
binding's checks see them."""
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


def codes(*shape, dtype=torch.int8):
    return OnDevice(torch.zeros(*shape, dtype=dtype))


def test_codes_that_are_taken():
    M, N, W = 6, 70, 80         # rows of 80 bytes
    for t, ld, step in ((codes(M, W), None, W), (codes(M + 2, W), None, W), (codes(2, 3, W), None, W), (codes(M * W + 7), None, W),
                        (OnDevice(codes(M, W).t[:, :N]), None, W), (OnDevice(codes(M, 96).t[:, :N]), None, 96),
                        (OnDevice(codes(M, 96).t[:, :W]), None, 96), (codes(M * 96), 96, 96), (codes(M, 96), 96, 96),
                        (codes(M, W, dtype=torch.uint8), None, W)):
        p, got = args().codes(t, M, N, ld, "a")
        assert p == t.data_ptr() and got == step, tuple(t.shape)
    for t in (codes(1, W), OnDevice(codes(W).t[None, :N]), codes(1, 1, W), codes(W)):
        assert args().codes(t, 1, N, None, "a")[1] == W
    assert args().codes(codes(5, 64), 5, 64, None, "a")[1] == 64
    # calls of no values read nothing
    args().codes(codes(0), 0, N, None, "a")
    args().codes(codes(4, 5), 4, 0, None, "a")
    assert args().codes(None, M, N, None, "a")[0] is None


def test_codes_that_are_refused():
    M, N = 6, 70
    for t, what in ((codes(M, N), "bytes apart"), (codes(M, 96), "rows of 70"), (codes(M, 64), "rows of 70"), (codes(M - 1, 80), "5 rows"),
                    (codes(80, M), "rows of 70"), (OnDevice(codes(80, M).t.t()), "unit stride"), (codes(M * 80 - 1), "contiguous codes"),
                    (OnDevice(codes(2, 3, 96).t[:, :, :N]), "contiguous"), (OnDevice(codes(M, 80).t[:, 10:]), "behind the tensor"),
                    (codes(M, 80, dtype=torch.int16), "8-bit"), (codes(M, 80, dtype=torch.float32), "8-bit")):
        with pytest.raises(ValueError, match=what):
            args().codes(t, M, N, None, "a")
    with pytest.raises(ValueError, match="contiguous codes"):
        args().codes(codes(M * 96 - 17), M, N, 96, "a")
    with pytest.raises(ValueError, match="unit stride"):
        args().codes(OnDevice(codes(2 * M, 160).t[:M, ::2]), M, N, None, "a")
