"""Layers in 8 bits: how near the codes of a norm are to the formula's, and products whose workspace is not given."""
import numpy as np
import pytest
import torch

import linear8_plan
import paper_2509_22323_amd as ra
from layer_common import normal, widen
from test_gpu_int8 import codes, scales

pytestmark = pytest.mark.gpu


def normed(x, scale, shift, eps):
    """(y, R) in 64-bit mantissas: R = max |1 + scale| (|x - mean| + mean |x|) / sqrt(variance + eps), against max |y|"""
    x, scale, shift = (np.asarray(t, np.longdouble) for t in (x, scale, shift))
    off = x - x.mean(-1, keepdims=True)
    by = (1 + scale) / np.sqrt((off * off).mean(-1, keepdims=True) + np.longdouble(np.float32(eps)))
    y = off * by + shift
    return y, (np.abs(by) * (np.abs(off) + np.abs(x).mean(-1, keepdims=True))).max(-1) / np.abs(y).max(-1)


@pytest.mark.parametrize("C", [64, 1536, 2432, 4096, 6144, 9728, 16384])
@pytest.mark.parametrize("kind", ["plain", "around", "far", "one", "undone"])
def test_codes_are_the_formulas(C, kind):
    """Half a step, and 2^-43 + 2^-39 R.  With u = 2^-53: a sum of the row is 58 additions deep at most, so the mean is off by 58 u mean |x|, and the
    deviation's reciprocal by 29 u for its sum, 4 u for the root and 3 u; an element of the norm is off by 58 u |1 + scale| (|x - mean| +
    mean |x|) / sqrt(variance + eps) in all, that is 58 u R max |y|, and by u |y|; so is the largest, and the quotient by 5 u more:
    127 (116 u R + 7 u) < 2^-39 R + 2^-43 (what this test computes it from is 2^-11 of that off)."""
    n = 24
    x, scale, shift = normal((1, n, C), C, 3.0), normal((1, C), C + 1, 0.3), normal((1, C), C + 2, 0.3)
    if kind == "around":
        x, scale, shift = normal((1, n, C), C, 1.0, 0.5), 0 * scale, 0 * shift
    if kind == "far":
        x = normal((1, n, C), C, 3.0, 300.0)
    if kind == "one":
        x[:] = 300.0
        for i in range(n):
            x[0, i, (7 * i + 3) % C] = 302.0 + i
    if kind == "undone":                               # what a row's norm comes to, taken off it again
        x[:] = x[:, :1]
        shift = torch.from_numpy(-normed(widen(x)[0, :1], widen(scale), 0.0, 1e-6)[0].astype(np.float32)).to(torch.bfloat16).cuda()
    q, q_scale = ra.rapid_norm_modulate_int8(x, torch.zeros((1, n, C), dtype=torch.int8, device="cuda"), torch.zeros((1, n), device="cuda"), scale, shift)
    y, R = normed(widen(x)[0], widen(scale), widen(shift), 1e-6)
    m = np.abs(y).max(-1)
    assert (np.abs(widen(q)[0] - 127 * y / m[:, None]) <= 0.5 + 2.0 ** -43 + 2.0 ** -39 * R[:, None]).all()
    # (rounded once to fp32, of a maximum that is off by (58 R + 2) u)
    assert (np.abs(widen(q_scale)[0] - m / 127) <= (2.0 ** -24 * (1 + 2.0 ** -20) + 2.0 ** -47 * R) * m / 127).all()


@pytest.mark.parametrize("product", [p for p in linear8_plan.PRODUCTS if p[5] > 1], ids=str)
def test_without_a_workspace(product):
    """The C entry without one, where the plan would cut the product along K: the same bits"""
    B, n, K, N, _, _ = product
    x, w, xs, ws = codes((B, n, K), 1), codes((N, K), 2), scales((B, n), 3, 0.01), scales((N,), 4, 0.01)
    bias, residual = normal((N,), 5), normal((B, n, N), 7)
    assert ra.rapid_linear_int8_workspace_bytes(B * n, N, K) > 0
    want = ra.rapid_linear_int8(x, xs, w, ws, torch.empty((B, n, N), dtype=torch.bfloat16, device="cuda"), bias, "gelu_tanh", None, residual)
    got = torch.full_like(want, float("nan"))
    rows = [ra.binding._rows("", t, None, dtype)[0] for t, dtype in ((x, "int8"), (got, "bfloat16"), (residual, "bfloat16"))]
    status = ra.library().rapid_linear_int8(rows[0], xs.data_ptr(), w.data_ptr(), K, ws.data_ptr(), bias.data_ptr(), rows[1], 2, None, 0, rows[2], None, 0,
                                            B, n, N, K, None, 0, torch.cuda.current_stream().cuda_stream)
    assert status == 0 and torch.equal(got.view(torch.int16), want.view(torch.int16))
