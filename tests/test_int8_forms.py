"""That the sizes of the 8-bit products' GPU tests take the kernels and blocks that they are
there for, and that together they take every one that the rules can give, without a GPU."""
import random

import pytest

import int8_forms as forms


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    return forms.Rules(str(tmp_path_factory.mktemp("forms")))


@pytest.mark.parametrize("form,M,N,K,ldb", forms.PRODUCTS)
def test_products(rules, form, M, N, K, ldb):
    assert rules.product(M, N, K, ldb) == form


@pytest.mark.parametrize("form,T,K,E,N,H,gather,align,ldb", forms.EXPERTS)
def test_experts(rules, form, T, K, E, N, H, gather, align, ldb):
    rows = forms.expert_rows(T, K, E, align)
    assert rules.experts(rows, N, H, E, T if gather else rows, K, gather, ldb) == form


def test_longest_sums(rules):
    for form, M, N in forms.LONGEST:
        assert rules.product(M, N, 131071) == form, (M, N)
    for form, counts, N in forms.LONGEST_EXPERTS:
        assert rules.experts(sum(counts), N, 131071, len(counts), sum(counts), 1, False) == form, (counts, N)


def test_a_block_in_tiles(rules):
    T, K, E, H, F, Q = (forms.TILED_BLOCK[k] for k in "TKEHFQ")
    tiles = lambda m, n: -(-m // 256) * -(-n // 256)
    assert rules.product(T, Q, H) == "tile" and tiles(T, Q) > 256
    assert rules.experts(T * K, F, H, E, T, K, True) == "tile" and tiles(T * K, F) > 256
    assert rules.experts(T * K, H, F, E, T * K, 1, False) == "tile" and tiles(T * K, H) >= 256


def test_no_form_is_left_out(rules):
    """Every form of sizes spread over the whole range (over their logarithms)."""
    rng = random.Random(0)
    log = lambda lo, hi: int(round(2 ** rng.uniform(lo, hi)))
    lines = lambda n: -(-n // 128) * 128 if rng.random() < 0.7 else forms.row_bytes(n)
    products, experts = set(), set()
    for _ in range(60000):
        M, N, K = log(0, 15), log(0, 16), log(0, 17) - 1
        products.add(rules.product(M, N, K, lines(K)))
        T, k, E, N, H, gather = log(0, 14), rng.choice([1, 2, 4, 8]), log(0, 9), log(0, 14), log(0, 15), rng.random() < 0.5
        experts.add((rules.experts(T * k, N, H, E, T if gather else T * k, k, gather, lines(H)), gather))
    assert products == {p[0] for p in forms.PRODUCTS}
    assert experts == {(e[0], e[6]) for e in forms.EXPERTS}
