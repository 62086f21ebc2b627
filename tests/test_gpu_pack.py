"""8-bit checkpoints on the GPU: codes, scales and the values read back, bit for
bit as the reference has them (every step but the code's rounding is exact)."""
import itertools

import numpy as np
import pytest

import oracle
import paper_2504_19519_amd as fo
from gpu_util import say, torch_mod
from oracle import rowops as ref
from rowops_util import Mat

pytestmark = pytest.mark.gpu
BOTH = list(itertools.product(["fp16", "bf16"], ["int8", "e4m3"]))


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = torch_mod()
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    fo.lib()
    yield
    torch.cuda.synchronize()


def from_bits(bits, dtype, ld=None, shift=0):
    torch = torch_mod()
    m = Mat(*bits.shape, dtype, ld, shift)
    m.raw.as_strided(bits.shape, (m.ld, 1), shift).copy_(torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)))
    return m


def check(m, fmt, what):
    torch = torch_mod()
    say(f"[pack] {what} {m.M}x{m.N} {m.dtype} {fmt} ld={m.ld} shift={m.shift}")
    a, b = fo.packed_bytes(m.M, m.N)
    codes = torch.full((a + 16,), 99, dtype=torch.uint8, device="cuda")
    scales = torch.full((b + 16,), 99, dtype=torch.uint8, device="cuda")
    fo.pack_rows(m.t, codes, scales, m.M, m.N, m.dtype, fmt)
    out = Mat(m.M, m.N, m.dtype, m.ld, m.shift)
    fo.unpack_rows(codes, scales, out.t, m.M, m.N, m.dtype, fmt)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        c, s = ref.pack(m.values(), fmt, m.dtype)
    np.testing.assert_array_equal(scales.cpu().numpy(), np.concatenate([s.reshape(-1), np.full(16, 99, np.uint8)]), err_msg=what)
    np.testing.assert_array_equal(codes.cpu().numpy(), np.concatenate([c.reshape(-1), np.full(16, 99, np.uint8)]), err_msg=what)
    want = ref.unpack(c, s, m.N, fmt)
    nan = np.isnan(want)
    got = out.values()
    np.testing.assert_array_equal(np.isnan(got), nan, err_msg=what)
    stored = oracle.decode(oracle.encode(np.where(nan, 0, want), m.dtype), m.dtype)
    np.testing.assert_array_equal(got[~nan], stored[~nan], err_msg=what)
    assert out.guards_stand(), what


@pytest.mark.parametrize("dtype,fmt", BOTH)
def test_every_bit_pattern(dtype, fmt):
    """Each 16-bit pattern once in a row of neighbours, and each as the largest of a block."""
    bits = np.arange(65536, dtype=np.uint16)
    check(from_bits(bits.reshape(64, 1024), dtype), fmt, "in order")
    rng = np.random.default_rng(1)
    check(from_bits(rng.permutation(bits).reshape(128, 512), dtype), fmt, "mixed")
    top = np.arange(0x7C00 if dtype == "fp16" else 0x7F80, dtype=np.uint16)
    x = oracle.decode(top, dtype)[:, None] * rng.uniform(-1, 1, (len(top), 32)) * np.exp2(-rng.integers(0, 10, (len(top), 32)))
    block = oracle.encode(x, dtype)
    block[np.arange(len(top)), rng.integers(0, 32, len(top))] = top | 0x8000
    check(from_bits(block, dtype), fmt, "largest of a block")


@pytest.mark.parametrize("dtype,fmt", BOTH)
@pytest.mark.parametrize("N", [1, 7, 8, 31, 32, 33, 40, 65, 100, 504, 512, 520, 1001, 2880, 16384, 40000])
def test_lengths(dtype, fmt, N):
    rng = np.random.default_rng(N)
    for M in (1, 3, 10):
        check(from_bits(oracle.encode(rng.normal(size=(M, N)) * np.exp(rng.normal(size=(M, 1)) * 3), dtype), dtype), fmt, "length")


@pytest.mark.parametrize("N,ld,shift", [(33, 34, 1), (64, 64, 3), (100, 137, 5), (512, 1024, 8), (2880, 2881, 7)])
def test_strides_and_alignment(N, ld, shift):
    rng = np.random.default_rng(N)
    for dtype, fmt in BOTH:
        check(from_bits(oracle.encode(rng.normal(size=(6, N)), dtype), dtype, ld, shift), fmt, "strided")


def test_nothing():
    fo.pack_rows(None, None, None, 0, 64, "fp16")
    fo.unpack_rows(None, None, None, 4, 0, "fp16")


@pytest.mark.parametrize("dtype,fmt", [("fp16", "int8"), ("bf16", "e4m3")])
def test_past_4_gib(dtype, fmt):
    """Rows whose places pass 32 bits: the first and last rows of a 4.3 GB matrix."""
    torch = torch_mod()
    M, N = 65560, 32768
    say(f"[pack] {M}x{N} {dtype} {fmt}")
    x = torch.zeros(M, N, dtype=torch.float16 if dtype == "fp16" else torch.bfloat16, device="cuda")
    a, b = fo.packed_bytes(M, N)
    codes, scales = torch.empty(a, dtype=torch.uint8, device="cuda"), torch.empty(b, dtype=torch.uint8, device="cuda")
    x[:2] = torch.randn(2, N, device="cuda")
    x[-2:] = torch.randn(2, N, device="cuda")
    fo.pack_rows(x, codes, scales, M, N, dtype, fmt)
    out = torch.full_like(x, 3.0)
    fo.unpack_rows(codes, scales, out, M, N, dtype, fmt)
    torch.cuda.synchronize()
    for rows in (slice(0, 2), slice(M - 2, M)):
        v = x[rows].double().cpu().numpy()
        want = ref.unpack(*ref.pack(v, fmt, dtype), N, fmt)
        np.testing.assert_array_equal(out[rows].double().cpu().numpy(), oracle.decode(oracle.encode(want, dtype), dtype))
    assert not bool(out[2:-2].any())
