"""The oracle of layers in 8 bits over packed sequences against properties that the definitions have."""
from fractions import Fraction

import numpy as np

from oracle import layer_oracle as lo
from oracle import packed_oracle as po

RNG = np.random.default_rng(5)


def bf16(x):
    """x as bf16 values (cut, not rounded)"""
    return (np.asarray(x, np.float32).view(np.uint32) & 0xFFFF0000).view(np.float32).astype(np.float64)


def test_quantised_rows_are_the_nearest_multiples():
    x = bf16(RNG.standard_normal((40, 96)) * np.exp(RNG.uniform(-40, 40, (40, 1))))
    x[:, 0] = 2 * np.abs(x).max(-1)                                        # (halves of the largest: ties)
    x[:, 1] = x[:, 0] / 2
    q, scale = po.quantize(x)
    for row, codes, s in zip(x, q, scale):
        m = Fraction(np.abs(row).max())
        for v, c in zip(row, codes):
            exact = Fraction(v) * 127 / m
            assert abs(exact - int(c)) <= Fraction(1, 2)
            if abs(exact - int(c)) == Fraction(1, 2):
                assert int(c) % 2 == 0
        assert s == float(m) / 127 and np.abs(codes).max() == 127


def test_rows_of_zeros_and_of_what_is_no_number():
    q, scale = po.quantize(np.array([[0.0, -0.0], [1.0, np.inf], [np.nan, 1.0], [1.0, -2.0]]))
    assert (q[:3] == 0).all() and scale[0] == 0 and np.isnan(scale[1:3]).all() and (q[3] == [64, -127]).all()


def test_products_of_quantised_rows_are_near_the_products():
    x, w = RNG.standard_normal((2, 5, 64)), RNG.standard_normal((7, 64))
    (xq, xs), (wq, ws) = po.quantize(x), po.quantize(w)
    assert np.abs(po.linear(xq, xs, wq, ws) - lo.linear(x, w)).max() < 64 * (xs.max() * np.abs(w).max() + ws.max() * np.abs(x).max())
    document = np.array([[0, 1, 1, -1, 0], [2, 2, 0, 1, 1]])
    g = RNG.standard_normal((3, 7))
    y = po.linear(xq, xs, wq, ws, gate=g, document=document)
    assert np.allclose(y[1, 0], po.linear(xq, xs, wq, ws)[1, 0] * g[2])
    s, t = RNG.standard_normal((2, 3, 64))
    n = po.norm_modulate(x, s, t, document=document)
    assert np.allclose(n[0, 1:3], lo.norm_modulate(x, np.stack([s[1]] * 2), np.stack([t[1]] * 2))[0, 1:3])


def test_packed_documents_are_what_each_is_alone():
    B, H, N, D = 2, 2, 23, 8
    q, k, v = RNG.standard_normal((3, B, H, N, D))
    document = np.stack([RNG.permutation(np.array([0] * 7 + [1] * 1 + [5] * 11 + [-1] * 4)) for _ in range(B)])
    for cap in (0.0, 2.0):
        o, p = po.attention(q, k, v, document, cap=cap)
        for b in range(B):
            for d in (0, 1, 5):
                at = document[b] == d
                s = q[b][:, at] @ np.swapaxes(k[b][:, at], 1, 2) / np.sqrt(D)
                s = cap * np.tanh(s / cap) if cap else s
                e = np.exp(s)
                assert np.allclose(o[b][:, at], e @ v[b][:, at] / e.sum(-1, keepdims=True))
            assert (o[b][:, document[b] < 0] == 0).all()
        assert np.allclose(p.sum(-1), (document >= 0)[:, None])


def test_orders():
    document = np.zeros((1, 6), int)
    causal = po.visible(document, np.arange(6)[None])
    assert (causal[0] == np.tril(np.ones((6, 6), bool))).all()
    prefix = po.visible(document, np.array([[0, 0, 0, 1, 2, 3]]))[0]
    assert prefix[:3, :3].all() and not prefix[:3, 3:].any() and (prefix[3:] == np.tril(np.ones((6, 6), bool))[3:]).all()
    text_first = po.visible(document, np.array([[1, 1, 1, 1, 0, 0]]))[0]
    assert text_first[:4].all() and (text_first[4:] == [0, 0, 0, 0, 1, 1]).all()
    assert po.visible(document, -np.arange(6)[None])[0].diagonal().all()


def test_what_is_not_visible_has_no_part():
    q, k, v = RNG.standard_normal((3, 1, 1, 8, 4))
    document = np.array([[0, 0, 0, 1, 1, -1, 0, 1]])
    want, _ = po.attention(q, k, v, document)
    k2, v2 = k.copy(), v.copy()
    k2[..., 5, :], v2[..., 5, :] = np.nan, np.inf
    v2[..., 3, 1] = np.nan
    got, _ = po.attention(q, k2, v2, document)
    mine = document[0] == 0
    assert np.allclose(got[0, 0, mine], want[0, 0, mine]) and np.isnan(got[0, 0, document[0] == 1, 1]).all()
