"""Products of 8-bit matrices in every kernel and every form of blocks (tests/int8_forms.py: the
sizes, and that they take these forms), whole sizes and ragged ones, all results against sums
in 64 bits on the GPU."""
import pytest

import int8_forms as forms
import paper_2504_19519_amd as fo
from gpu_util import say, torch_mod
from int8_util import Codes
from rowops_util import F32, HALF, TINY, Mat, torch_dtype

pytestmark = pytest.mark.gpu
DTYPES = ["fp16", "bf16"]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = torch_mod()
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    fo.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def draw(gen, rows, K, ld):
    """Codes in rows `ld` apart, zeros behind a row's end up to its whole chunks of 16, a pattern behind those."""
    torch = torch_mod()
    m = Codes(rows, K, ld)
    m.whole.zero_()
    m.t.copy_(torch.randint(-128, 128, (rows, K), generator=gen, dtype=torch.int8, device="cuda"))
    return m


def check(C, rows, a, sa, b, sb, bias, dtype, what):
    """Rows of C against a b^T sa sb + bias. The sums are exact in 64 bits; the kernel's is rounded to 32, as are two
    products and the bias's addition; then once to 16."""
    torch = torch_mod()
    right = b.double().t().contiguous()
    for lo in range(0, len(rows), 1024):
        at = rows[lo:lo + 1024]
        want = (a[lo:lo + 1024].double() @ right) * sa[lo:lo + 1024].double()[:, None] * sb.double()
        mag = want.abs()
        if bias is not None:
            want = want + bias.double()
        extra = 3 * F32 * mag + F32 * want.abs()
        off = (C.t[at].double() - want).abs() - (HALF[dtype] * (want.abs() + extra) + TINY[dtype] + extra)
        assert bool((off <= 0).all()), (what, int((off > 0).sum()), "first at row", int(at[0]) + int((off > 0).any(1).int().argmax()))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("form,M,N,K,ldb", forms.PRODUCTS)
def test_product(form, M, N, K, ldb, dtype):
    torch = torch_mod()
    say(f"[int8 forms] {form}: {M}x{N}x{K} {dtype}")
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    # (rows of c at every alignment: odd distances, one value into the allocation, in one of the types)
    odd = dtype == "fp16"
    A, B, C = draw(gen, M, K, None), draw(gen, N, K, ldb), Mat(M, N, dtype, N + 3 if odd else None, 1 if odd else 0)
    sa, sb = (torch.exp2(-9 + 4 * torch.rand(n, generator=gen, device="cuda")) for n in (M, N))
    bias = torch.randn(N, generator=gen, device="cuda").to(torch_dtype(dtype)) if (M + odd) % 2 else None
    work = torch.full((fo.int8_workspace_bytes(M, N, K),), 0xFF, dtype=torch.uint8, device="cuda")
    assert (len(work) > 0) == ("parts" in form)
    fo.int8_product(A.whole, sa, B.whole, sb, C.t, M, N, K, dtype, bias=bias, workspace=work)
    check(C, torch.arange(M, device="cuda"), A.t, sa, B.t, sb, bias, dtype, form)
    assert C.guards_stand()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("form,T,K,E,N,H,gather,align,ldb", forms.EXPERTS)
def test_experts(form, T, K, E, N, H, gather, align, ldb, dtype):
    torch = torch_mod()
    say(f"[int8 forms] {form}: {T} tokens to {K} of {E}, {N}x{H} {dtype}")
    assert fo.route_capacity(T, K, E, align) == forms.expert_rows(T, K, E, align)
    gen = torch.Generator(device="cuda").manual_seed(T + N + H)
    cap, odd = forms.expert_rows(T, K, E, align), dtype == "bf16"
    rows = T if gather else cap
    # (experts of uneven size, some choices dropped)
    ids = torch.topk(torch.randn(T, E, generator=gen, device="cuda") + torch.randn(E, generator=gen, device="cuda"), K, dim=1)[1]
    ids = torch.where(torch.rand(T, K, generator=gen, device="cuda") < 0.03, -1, ids).to(torch.int32)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    offsets, counts, slot, pairs = i32(E + 1), i32(E), i32(T * K), i32(cap)
    sort = torch.empty(fo.route_workspace_bytes(T, K, E), dtype=torch.uint8, device="cuda")
    fo.route_sort(ids, T, K, E, offsets, counts, slot, pairs, sort, align)
    A, B, C = draw(gen, rows, H, None), draw(gen, E * N, H, ldb), Mat(cap, N, dtype, N + 1 if odd else None)
    sa, sb = (torch.exp2(-9 + 4 * torch.rand(n, generator=gen, device="cuda")) for n in (rows, E * N))
    bias = torch.randn(E * N, generator=gen, device="cuda").to(torch_dtype(dtype)) if (T + odd) % 2 else None
    fo.int8_experts(A.whole, sa, B.whole, sb, C.t, N, H, E, dtype, cap, offsets, counts, rows, pair_of=pairs if gather else None,
                    choices=K, bias=bias)
    written = []
    for e, (at, n) in enumerate(zip(offsets.tolist(), counts.tolist())):
        if n == 0:
            continue
        c = torch.arange(at, at + n, device="cuda")
        src = pairs[c].long() // K if gather else c
        w = slice(e * N, (e + 1) * N)
        check(C, c, A.t[src], sa[src], B.t[w], sb[w], None if bias is None else bias[w], dtype, (form, e))
        written += list(range(at, at + n))
    assert len(written) == int((ids >= 0).sum()) and C.guards_stand(written)


def test_the_reference_sees_a_wrong_sum():
    """One product too many in one place: outside the bound."""
    torch = torch_mod()
    gen = torch.Generator(device="cuda").manual_seed(1)
    A, B, C = draw(gen, 70, 200, None), draw(gen, 60, 200, None), Mat(70, 60, "fp16")
    s = torch.full((70,), 2.0 ** -7, device="cuda")
    fo.int8_product(A.whole, s, B.whole, s[:60], C.t, 70, 60, 200, "fp16")
    rows = torch.arange(70, device="cuda")
    check(C, rows, A.t, s, B.t, s[:60], None, "fp16", "as it is")
    a = A.t.clone()
    a[33, 7] += -100 if int(a[33, 7]) > 0 else 100
    with pytest.raises(AssertionError):
        check(C, rows, a, s, B.t, s[:60], None, "fp16", "another operand")
