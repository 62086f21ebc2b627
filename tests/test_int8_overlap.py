"""What the norm's backward pass of a sum writes and what it reads, in one piece of memory:
refused without a GPU, where the description does not allow it."""
import pytest

import paper_2504_19519_amd as fo

P = 1 << 24          # stands for device memory; no refused call gets as far as using it
ARG = -1


def status(f, *args, **kw):
    """That a call fails with. (A call that is taken fails at its launch where there is no GPU.)"""
    with pytest.raises(fo.FoError) as e:
        f(*args, **kw)
    return e.value.status


def backward(dy=P, dh=2 * P, h=3 * P, gamma=4 * P, rstd=5 * P, dx=6 * P, dgamma=7 * P, workspace=8 * P, M=4, N=64, **kw):
    fo.norm_add_backward(dy, dh, h, gamma, rstd, dx, dgamma, M, N, "bf16", workspace, **kw)


ROWS = 4 * 64 * 2           # bytes of a matrix
END = object()              # the last 16 bytes of the workspace (whose size the library gives) begin there


@pytest.mark.parametrize("what,bad", [
    ("dx", dict(gamma=6 * P)), ("dx", dict(gamma=6 * P + ROWS - 2)), ("dx", dict(rstd=6 * P + 4)), ("dx", dict(dgamma=6 * P)),
    ("dx", dict(dgamma=6 * P - 4 * 64 + 4)), ("dx", dict(workspace=6 * P)), ("dx", dict(dx=END)),
    ("dgamma", dict(dgamma=P)), ("dgamma", dict(dgamma=2 * P + ROWS - 4)), ("dgamma", dict(dgamma=3 * P)),
    ("dgamma", dict(dgamma=4 * P)), ("dgamma", dict(dgamma=5 * P + 12)), ("dgamma", dict(dgamma=8 * P)),
    ("dgamma", dict(dgamma=END)), ("dgamma", dict(dx=None, dgamma=P)),
    ("workspace", dict(workspace=P)), ("workspace", dict(workspace=2 * P)), ("workspace", dict(workspace=3 * P + ROWS - 16)),
    ("workspace", dict(workspace=4 * P)), ("workspace", dict(workspace=5 * P)),
    ("workspace", dict(dx=None, workspace=3 * P)),
])
def test_refused(what, bad):
    end = 8 * P + fo.norm_workspace_bytes(4, 64) - 16
    assert status(backward, **{k: end if v is END else v for k, v in bad.items()}) == ARG
    assert what in fo.lib().fo_last_error().decode()


def test_rows_too_wide_to_be_held_have_a_workspace_without_dgamma():
    wide = dict(M=2, N=20000, dgamma=None, gamma=None)
    for at in (P, 2 * P, 3 * P, 5 * P, 6 * P):
        assert status(backward, workspace=at, **wide) == ARG, at


@pytest.mark.parametrize("good", [dict(dx=P), dict(dx=2 * P), dict(dx=3 * P), dict(dh=None), dict(dgamma=None, workspace=None),
                                  dict(dgamma=None, workspace=P),           # (not used)
                                  dict(dx=None, dgamma=2 * P),              # (dh is not read)
                                  dict(dy=P, dh=P, h=P, dx=P),
                                  # side by side, to the byte
                                  dict(dx=6 * P, dgamma=6 * P + ROWS), dict(gamma=6 * P - 128), dict(rstd=6 * P + ROWS),
                                  dict(workspace=6 * P + ROWS), dict(dgamma=8 * P - 256), dict(workspace=7 * P + 256)], ids=str)
def test_taken(good):
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("the pointers stand for no memory: without a GPU only")
    assert status(backward, **good) not in (ARG, -2, -3)


def test_no_rows_are_no_overlap():
    """Nothing is read then, and dgamma alone written: neither input nor workspace is looked at."""
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("the pointers stand for no memory: without a GPU only")
    assert status(backward, M=0, dgamma=P, workspace=None) not in (ARG, -2, -3)
