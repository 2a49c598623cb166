"""The oracle of the operators around the attention against properties that the definitions have."""
import math

import numpy as np
import pytest

from oracle import layer_oracle as lo

RNG = np.random.default_rng(3)


def test_activations():
    z = RNG.standard_normal(1000) * 4
    phi = np.array([0.5 * (1.0 + math.erf(v / math.sqrt(2.0))) for v in z])
    assert np.abs(lo.activation(z, "gelu_tanh") - z * phi).max() < 5e-4            # the known distance of the two forms
    assert np.allclose(lo.activation(z, "silu") - lo.activation(-z, "silu"), z)     # sigma(z) + sigma(-z) = 1
    assert np.allclose(lo.activation(z, "gelu_tanh") - lo.activation(-z, "gelu_tanh"), z)


def test_linear_is_linear_and_gated_by_sample():
    x, w, b = RNG.standard_normal((2, 3, 8)), RNG.standard_normal((5, 8)), RNG.standard_normal(5)
    want = np.einsum("bnk,jk->bnj", x, w) + b
    assert np.allclose(lo.linear(x, w, b), want)
    g, r = RNG.standard_normal((2, 5)), RNG.standard_normal((2, 3, 5))
    assert np.allclose(lo.linear(x, w, b, "none", g, r)[1], want[1] * g[1] + r[1])


def test_norms():
    x = RNG.standard_normal((2, 4, 64)) * 3 + 7
    y = lo.norm_modulate(x, eps=0.0)
    assert np.allclose(y.mean(-1), 0) and np.allclose((y * y).mean(-1), 1)
    assert np.allclose(lo.norm_modulate(5 * x + 3, eps=0.0), y)
    s, t = RNG.standard_normal((2, 64)), RNG.standard_normal((2, 64))
    assert np.allclose(lo.norm_modulate(x, s, t, 0.0)[1], y[1] * (1 + s[1]) + t[1])
    u = lo.head_norm(x, eps=0.0)
    assert np.allclose((u * u).mean(-1), 1) and np.allclose(lo.head_norm(9 * x, eps=0.0), u)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("rot", [16, 48, 64])
def test_scores_of_turned_rows_depend_on_the_distance_alone(layout, rot):
    p = np.arange(40)[:, None]
    table = lo.table(p, [dict(dim=rot, theta=100.0)])
    q, k = np.broadcast_to(RNG.standard_normal((2, 1, 1, 1, 64)), (2, 1, 1, 40, 64))
    a, b = lo.rotate(q, table, layout)[0, 0], lo.rotate(k, table, layout)[0, 0]
    s = a @ b.T
    assert np.allclose(s[5, 12], s[20, 27]) and np.allclose(s[30, 3], s[36, 9]) and not np.allclose(s[5, 12], s[5, 13])
    assert np.allclose(np.linalg.norm(a, axis=-1), np.linalg.norm(q[0, 0], axis=-1))


def test_layouts_are_the_same_up_to_the_order_of_elements():
    v, table = RNG.standard_normal((1, 2, 7, 64)), lo.table(np.arange(7)[:, None], [dict(dim=64, theta=50.0)])
    order = np.concatenate([np.arange(0, 64, 2), np.arange(1, 64, 2)])
    assert np.allclose(lo.rotate(v, table, "interleaved")[..., order], lo.rotate(v[..., order], table, "half"))


def test_frequencies_and_scalings():
    d, s = 64, 4.0
    f = lo.frequencies(d, 10000.0)
    assert f[0] == 1.0 and np.isclose(f[-1], 10000.0 ** (-62 / 64)) and (np.diff(f) < 0).all()
    assert np.allclose(lo.frequencies(d, 10000.0, "linear", s), f / s)
    n = lo.frequencies(d, 10000.0, "ntk", s)
    assert n[0] == f[0] and np.isclose(n[-1], f[-1] / s)                            # the fastest kept, the slowest by the factor
    p = lo.frequencies(d, 10000.0, "by_parts", s, 4096.0, 32.0, 1.0)
    turns = 4096.0 * f / (2 * math.pi)
    assert np.allclose(p[turns > 32], f[turns > 32]) and np.allclose(p[turns < 1], f[turns < 1] / s)
    assert ((p <= f) & (p >= f / s)).all() and (turns > 32).any() and (turns < 1).any()


def test_axes_of_the_table():
    p = np.stack([np.zeros(6), np.arange(6), 10 * np.arange(6)], -1).astype(np.int64)
    t = lo.table(p, [dict(dim=16, theta=10000.0), dict(dim=24, theta=10000.0), dict(dim=8, theta=10000.0)], 2.0)
    assert t.shape == (6, 24, 2) and np.allclose(t[:, :8], [2.0, 0.0])
    assert np.allclose(t[3, 8], [2 * math.cos(3.0), 2 * math.sin(3.0)]) and np.allclose(t[3, 20], [2 * math.cos(30.0), 2 * math.sin(30.0)])
