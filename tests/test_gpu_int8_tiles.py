"""rapid_linear_int8 in every tile and number of pieces, bare and with every part of its epilogue."""
import pytest

import linear8_plan
from test_gpu_int8 import check

pytestmark = pytest.mark.gpu

PARTS = [dict(bias=False), dict(act="gelu_tanh"), dict(gate=True, residual=True, in_place=True), dict(act="silu", gate=True, lengths=True, residual=True)]


@pytest.mark.parametrize("product", linear8_plan.PRODUCTS, ids=str)
def test_products(product):
    B, n, K, N, tile, pieces = product
    small = B * n * K * N < 2e9
    at = linear8_plan.PRODUCTS.index(product)
    for parts in PARTS if small else (PARTS[at % 4], PARTS[(at + 1) % 4]):
        kw = dict(parts)
        if kw.pop("lengths", False):
            kw["lengths"] = (n // 3, 1, n // 2)
        check(B, n, K, N, seed=at, **kw)


@pytest.mark.parametrize("product", [p for p in linear8_plan.PRODUCTS if p[0] * p[1] * p[2] * p[3] < 8e9 and p[5] == 1], ids=str)
def test_documents_in_the_large_tiles(product):
    B, n, K, N, _, _ = product
    check(B, n, K, N, act="none", gate=True, residual=True, lengths=(n // 2, n // 4, 3), seed=3)
