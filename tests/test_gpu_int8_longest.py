"""The longest sums (K = 131071) of every kernel and form: up to 2^31 - 2^14 in one accumulator
where k is not divided, over rows of one value and over rows whose values change from one k to
the next. The sums of the few distinct rows are exact in 64 bits; every result is checked."""
import pytest

import int8_forms as forms
import paper_2504_19519_amd as fo
from gpu_util import say, torch_mod
from rowops_util import F32, HALF, TINY, Mat

pytestmark = pytest.mark.gpu
K, W = 131071, 131072


@pytest.fixture(scope="module", autouse=True)
def gpu():
    torch = torch_mod()
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    fo.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def patterns():
    """(a's rows, b's rows, their sums): -128 and 127 throughout; both in random order, the same in a and in b, and
    with every sign turned but for a few; random codes; ones in one place only, the sum's last and first."""
    torch = torch_mod()
    gen = torch.Generator(device="cuda").manual_seed(3)
    code = lambda v: torch.full((K,), v, device="cuda")
    mixed = torch.where(torch.rand(K, generator=gen, device="cuda") < 0.5, -128, 127)
    a = [code(-128), code(127), mixed, torch.randint(-128, 128, (K,), generator=gen, device="cuda"), torch.zeros(K, device="cuda")]
    b = [code(-128), code(127), mixed, -1 - mixed, torch.randint(-128, 128, (K,), generator=gen, device="cuda")]
    a[4] = a[4].clone()
    a[4][K - 1] = 127
    a.append(torch.zeros(K, device="cuda"))
    a[5][0] = -128
    b.append(torch.arange(K, device="cuda") % 251 - 125)
    pad = lambda rows: torch.nn.functional.pad(torch.stack([r.to(torch.int8) for r in rows]), (0, W - K)).contiguous()
    a, b = pad(a), pad(b)
    sums = a.double() @ b.double().t().contiguous()
    assert float(sums.max()) == 2.0 ** 31 - 2.0 ** 14 and float(sums.min()) == -127.0 * 128 * K
    return a, b, sums


def rows(gen, n, of):
    """n rows, which of `of` each is."""
    torch = torch_mod()
    which = torch.randint(0, len(of), (n,), generator=gen, device="cuda")
    which[:min(n, len(of))] = torch.arange(min(n, len(of)), device="cuda")
    return of[which], which


def scales(gen, n, base):
    torch = torch_mod()
    return torch.exp2(base + torch.rand(n, generator=gen, device="cuda"))


def within(got, want, dtype, what):
    extra = 3 * F32 * want.abs()            # the sum in 32 bits, two products
    off = (got.double() - want).abs() - (HALF[dtype] * (want.abs() + extra) + TINY[dtype] + extra)
    assert bool((off <= 0).all()), (what, off.flatten().argmax().item(), int((off > 0).sum()))


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("form,M,N", forms.LONGEST)
def test_product(form, M, N, dtype):
    torch = torch_mod()
    say(f"[int8 longest] {form}: {M}x{N} {dtype}")
    gen = torch.Generator(device="cuda").manual_seed(M)
    pa, pb, sums = patterns()
    (a, wa), (b, wb) = rows(gen, M, pa), rows(gen, N, pb)
    sa, sb, C = scales(gen, M, -12), scales(gen, N, -8), Mat(M, N, dtype)
    work = torch.full((fo.int8_workspace_bytes(M, N, K),), 0xFF, dtype=torch.uint8, device="cuda")
    fo.int8_product(a, sa, b, sb, C.t, M, N, K, dtype, workspace=work)
    within(C.t, sums[wa][:, wb] * sa.double()[:, None] * sb.double(), dtype, form)
    assert C.guards_stand()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("form,counts,N", forms.LONGEST_EXPERTS)
def test_experts(form, counts, N, dtype):
    torch = torch_mod()
    say(f"[int8 longest] experts {form}: {counts} {N} {dtype}")
    gen = torch.Generator(device="cuda").manual_seed(N)
    pa, pb, sums = patterns()
    E, M = len(counts), sum(counts)
    (a, wa), (b, wb) = rows(gen, M, pa), rows(gen, E * N, pb)
    sa, sb, C = scales(gen, M, -12), scales(gen, E * N, -8), Mat(M, N, dtype)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    offsets = [sum(counts[:e]) for e in range(E + 1)]
    fo.int8_experts(a, sa, b, sb, C.t, N, K, E, dtype, M, i32(offsets), i32(counts), M)
    for e, n in enumerate(counts):
        r, w = slice(offsets[e], offsets[e] + n), slice(e * N, (e + 1) * N)
        if n:
            within(C.t[r], sums[wa[r]][:, wb[w]] * sa[r].double()[:, None] * sb[w].double(), dtype, (form, e))
    assert C.guards_stand()
