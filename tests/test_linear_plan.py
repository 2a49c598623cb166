"""The host's choice of a product's kernel: what the products of the GPU tests are taken in (so that other costs cannot silently leave a
tile untested), and its rules at the ends of their ranges.  No GPU needed."""
import math
import os

import pytest

import linear_plan
import paper_2509_22323_amd as ra
from paper_2509_22323_amd import build


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return linear_plan.load(tmp_path_factory.mktemp("plan"))


@pytest.mark.parametrize("product", linear_plan.PRODUCTS, ids=str)
def test_the_products_of_the_gpu_tests_are_taken_in_their_tiles(plan, product):
    B, n, K, N, tile, pieces = product
    got = plan(B * n, N, K)
    assert got == (tile, pieces) or tile == "" or (tile, got[1]) == ("dots", 0)


def test_the_products_of_the_gpu_tests_reach_every_form():
    one = {tile: {B == 1 for B, n, K, N, t, pieces in linear_plan.PRODUCTS if (t, pieces) == (tile, 1)} for tile in linear_plan.TILES}
    assert all(v == {False, True} for v in one.values()), one
    for tile in linear_plan.TILES[:2]:
        assert {pieces for *_, t, pieces in linear_plan.PRODUCTS if t == tile} == set(range(1, 9))


def test_workspaces_are_those_of_the_plan(plan):
    for B, n, K, N, _, _ in linear_plan.PRODUCTS:
        pieces = plan(B * n, N, K)[1]
        assert ra.rapid_linear_workspace_bytes(B * n, N, K) == (4 * pieces * B * n * -(-N // 8) * 8 if pieces > 1 else 0)
        assert plan(B * n, N, K, 1)[1] <= 1


@pytest.mark.parametrize("M", [1, 8, 9, 64, 1000, 32768, (1 << 31) - 257])
@pytest.mark.parametrize("N", [1, 7, 64, 2432, 1 << 22])
@pytest.mark.parametrize("K", [8, 64, 576, 9728, 1 << 22])
def test_any_size_has_a_plan(plan, M, N, K):
    tile, pieces = plan(M, N, K)
    assert tile == "dots" and M <= 8 or 1 <= pieces <= 8 and (pieces == 1 or 3 * pieces * 64 <= K and M * N < 1 << 31)


def timed():
    """(rows, outputs, inputs, us of the library, us of each form) of the products that were timed in every form"""
    path = os.path.join(os.path.dirname(build.HERE), "profiles", "linear_tiles.txt")
    forms = [(t, p) for t in linear_plan.TILES[:2] for p in range(1, 9)] + [(t, 1) for t in linear_plan.TILES[2:]]
    for line in open(path):
        if line[0].isdigit():
            m, n, k, library, *times = line.split()
            yield int(m), int(n), int(k), float(library), {f: float(t) for f, t in zip(forms, times, strict=True) if t != "-"}


@pytest.mark.parametrize("wide", [False, True])
def test_the_plan_costs_little_over_the_best_form(plan, wide):
    """In the times that are committed beside the costs: 1.01 in the geometric mean, of products within the fit's range and beyond it, and
    no more than the comment on the costs says."""
    over = []
    for m, n, k, _, times in timed():
        if (max(n, k) > 9728) == wide:
            over.append(times[plan(m, n, k)] / min(times.values()))
    assert len(over) == (100 if wide else 700)
    assert math.exp(sum(map(math.log, over)) / len(over)) <= 1.015 and max(over) <= (1.15 if wide else 1.4)
