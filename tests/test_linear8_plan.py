"""Which kernel a product of 8-bit integers is taken in; no GPU needed."""
import pytest

import linear8_plan
import paper_2509_22323_amd as ra


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return linear8_plan.load(tmp_path_factory.mktemp("plan"))


@pytest.mark.parametrize("product", linear8_plan.PRODUCTS, ids=str)
def test_the_products_of_the_gpu_tests_are_taken_in_their_tiles(plan, product):
    B, n, K, N, tile, pieces = product
    assert plan(B * n, N, K) == (tile, pieces)
    assert ra.rapid_linear_int8_workspace_bytes(B * n, N, K) == (0 if pieces == 1 else pieces * B * n * ((N + 7) // 8 * 8) * 4)


def test_every_form_has_a_product():
    forms = {p[4:] for p in linear8_plan.PRODUCTS}
    assert forms == {(t, 1) for t in linear8_plan.TILES[1:]} | {(t, pieces) for t in linear8_plan.TILES[:2] for pieces in range(2, 9)}


def test_a_handful_of_rows_is_taken_by_dots(plan):
    for M, N, K in ((1, 9216, 1536), (4, 12288, 6144), (8, 8192, 4096)):
        assert plan(M, N, K)[0] == "dots" and ra.rapid_linear_int8_workspace_bytes(M, N, K) == 0
    assert plan(8, 12288, 6144)[0] != "dots" and plan(9, 64, 64)[0] != "dots"
