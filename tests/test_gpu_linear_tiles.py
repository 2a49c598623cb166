"""rapid_linear in every tile and every number of pieces along K, in each form of its epilogue: products of whole numbers, whose sums
are exact in fp32 in any order, and random ones, nearly all of which have to round as the exact product does."""
import math

import numpy as np
import pytest
import torch

import paper_2509_22323_amd as ra
from layer_common import NAN, inside, untouched_around
from linear_plan import PRODUCTS
from oracle import layer_oracle as lo
from test_gpu_linear import assert_within, bound, widen

pytestmark = pytest.mark.gpu

CASES = [p[:4] for p in PRODUCTS]


def whole(g, low, high, *shape):
    return torch.randint(low, high + 1, shape, generator=g, device="cuda").to(torch.bfloat16)


def outputs(B, n, N, columns):
    """An output among NaN: whole rows side by side, or with `columns` more between them."""
    return inside(torch.full((B, n, N), NAN, dtype=torch.bfloat16, device="cuda"), 1, 1, columns)


def product(x, w):
    """fp64, on the GPU: exact for whole numbers, to 1e-16 of the absolute sums for others"""
    return (x.reshape(-1, x.shape[-1]).double() @ w.double().t()).view(*x.shape[:2], -1)


@pytest.mark.parametrize("columns", [0, 4, 3])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_whole_numbers(case, columns):
    """Sums stay below 2^24 and every operand of the epilogue is a whole number (gates: halves), so that fp32 holds each step of
    them and the one rounding to bf16 is the only one.  columns 0 and 4: rows at even elements, 3: at odd ones, too."""
    B, n, K, N = case
    g = torch.Generator("cuda").manual_seed(sum(case))
    x, w, b = whole(g, -8, 8, B, n, K), whole(g, -8, 8, N, K), whole(g, -200, 200, N)
    gate, res = whole(g, -4, 4, B, N) / 2, whole(g, -200, 200, B, n, N)
    sums = product(x, w)
    assert 4 * (sums.abs().max() + 200) + 200 < 1 << 23
    bare, gated = (sums + b.double()), (sums + b.double()) * gate.double()[:, None] + res.double()
    for want, args in ((bare, (b,)), (sums, ()), (gated, (b, "none", gate, res)), (gated - res.double(), (b, "none", gate)),
                       (bare + res.double(), (b, "none", None, res))):
        out, big = outputs(B, n, N, columns)
        ra.rapid_linear(x, w, out, *args)
        assert torch.equal(out, want.to(torch.bfloat16)) and untouched_around(out, big), len(args)
    out, big = outputs(B, n, N, columns)
    out.copy_(res)
    ra.rapid_linear(x, w, out, b, "none", gate, out)                               # in place
    assert torch.equal(out, gated.to(torch.bfloat16)) and untouched_around(out, big)


def differently_rounded(K):
    """What share of the outputs may round to another bf16 than the exact ones, which have variance 1.  A sum of K products takes
    K / 16 additions at least of partial sums below 4 deviations, each off by 2^-23 of them; independent, they make e = sqrt(K / 16)
    2^-21.  An output y is rounded differently where it lies within e of a border, borders being 2^-8 |y| apart or more: a share of
    c / |y| with c = 2^9 e at most, or all of them below |y| = c.  The density is at most 0.4 on either side: 0.8 c (1 + ln(1 / c))."""
    c = 2.0 ** 9 * math.sqrt(K / 16) * 2.0 ** -21
    return 0.8 * c * (1 + math.log(1 / c))


@pytest.mark.parametrize("case", CASES, ids=str)
def test_random_products_round_as_the_exact_ones(case):
    B, n, K, N = case
    g = torch.Generator("cuda").manual_seed(sum(case) + 1)
    x, w = (torch.randn(s, generator=g, device="cuda") for s in ((B, n, K), (N, K)))
    x, w = x.to(torch.bfloat16), (w * K ** -0.5).to(torch.bfloat16)
    out, big = outputs(B, n, N, 0)
    ra.rapid_linear(x, w, out)
    want = product(x, w)
    others = (out != want.to(torch.float32).to(torch.bfloat16)).double().mean().item()
    count = out.numel()
    # (five deviations of a share counted over this many outputs)
    p = differently_rounded(K)
    assert others <= p + 5 * math.sqrt(p / count) + 1 / count, (others, p)


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_activated_gated_and_added(case, act):
    """Activation, gate and residual of whole even rows, apart and in place, on rows of every kind of tile."""
    B, n, K, N = case
    g = torch.Generator("cuda").manual_seed(sum(case) + 2)

    def make(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16)

    x, w, b, gate, res = make(B, n, K), make(N, K, scale=K ** -0.5), make(N, scale=0.3), make(B, N), make(B, n, N)
    out, big = outputs(B, n, N, 0)
    ra.rapid_linear(x, w, out, b, act, gate, res)
    assert torch.isfinite(out).all() and untouched_around(out, big)
    same, _ = outputs(B, n, N, 0)
    same.copy_(res)
    assert torch.equal(ra.rapid_linear(x, w, same, b, act, gate, same), out)
    M = B * n
    m = np.unique(np.concatenate([[0, M - 1], np.random.default_rng(1).integers(0, M, 200), np.arange(max(0, M - 260), M, 37)]))
    s, r = torch.from_numpy(m // n).cuda(), torch.from_numpy(m % n).cuda()
    args = (widen(x[s, r])[:, None], widen(w), widen(b), act, widen(gate[s]), widen(res[s, r])[:, None])
    want = lo.linear(*args)
    assert_within(out[s, r][:, None], want, bound(*args, want), str(case))
