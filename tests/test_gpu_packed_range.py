"""rapid_attn_packed at the ends of its range: scores, caps, scales and values far from 1."""
import numpy as np
import pytest
import torch

import paper_2509_22323_amd as ra
from layer_common import BF16_STEP, NAN, assert_within, normal, widen
from oracle import packed_oracle as po
from test_gpu_attn_packed import bound, documents
from test_gpu_packed_calls import attend, form  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,H", [(200, 2), (1500, 1), (1500, 40)], ids=str)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("cap,scale,size", [(0.0, 0.0, 1e16), (1e32, 0.0, 1e16), (1e32, 1e30, 10.0)], ids=str)
def test_rows_whose_scores_are_all_far_below_zero(D, N, H, causal, cap, scale, size):
    """Scores of -10^32 and less, and no others, in some documents (a single token, three of equal scores, two of which one's is twice the
    other's) beside ordinary ones; in few tiles, in tiles that several workgroups share, and where a group has a workgroup to itself.
    Equal scores are equal weights, and the least of two such scores has none."""
    lengths = (70, 1, 3, 2, N - 100)
    d, at = documents(N, lengths), np.cumsum((0,) + lengths)
    order = np.arange(N, dtype=np.int32) if causal else None
    q, k, v = normal((3, 1, H, N, D), 3)
    if scale:                                          # (ordinary scores under it)
        q[:, :, :at[1]] *= scale ** -0.5 / 4
        k[:, :, :at[1]] *= scale ** -0.5 / 4
        q[:, :, at[4]:] *= scale ** -0.5 / 4
        k[:, :, at[4]:] *= scale ** -0.5 / 4
    q[:, :, at[1]:at[4]], k[:, :, at[1]:at[4]] = size, -size
    k[:, :, at[3] + 1] = -2 * size
    got = widen(attend(q, k, v, torch.from_numpy(d).cuda(), None if order is None else torch.from_numpy(order).cuda(), cap, scale))
    values = widen(v)
    assert np.isfinite(got).all() and not got[:, :, at[5]:].any()
    assert np.array_equal(got[:, :, at[1]], values[:, :, at[1]])
    for i in range(3):
        seen = values[:, :, at[2]:at[2] + (i + 1 if causal else 3)]
        assert (np.abs(got[:, :, at[2] + i] - seen.mean(2)) <= BF16_STEP * np.abs(seen.mean(2)) + 2.0 ** -21 * np.abs(seen).mean(2)).all()
    if not cap:
        assert np.array_equal(got[:, :, at[3]:at[4]], np.broadcast_to(values[:, :, at[3]:at[3] + 1], got[:, :, at[3]:at[4]].shape))
    if H < 40:
        s = scale if scale else D ** -0.5
        for a, z in ((0, at[1]), (at[4], at[5])):
            part = [widen(t)[:, :, a:z] for t in (q, k, v)]
            turn = None if order is None else order[None, a:z]
            o, p = po.attention(*part, d[None, a:z], turn, cap, s)
            # (a cap far above the scores costs them nothing but in proportion)
            assert (np.abs(got[:, :, a:z] - o) <= bound(*part, p, o, 0.0, s, po.visible(d[None, a:z], turn))).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N", [1, 64, 150, 1280])
def test_whole_tiles_far_below_zero(D, N):
    """One document, every score -8e32 or less: tiles that need no mask"""
    q, k, v = normal((3, 1, 1, N, D), 4)
    q[:], k[:] = 1e16, -1e16
    got = widen(attend(q, k, v, torch.zeros(N, dtype=torch.int32, device="cuda")))
    mean, size = widen(v).mean(2, keepdims=True), np.abs(widen(v)).mean(2, keepdims=True)
    assert (np.abs(got - mean) <= BF16_STEP * np.abs(mean) + (N + 2) * 2.0 ** -23 * size).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap,scale", [(1e14, 1e17), (1e5, 1e9), (1e30, 1e32)], ids=str)
def test_caps_under_which_a_power_series_leaves_fp32(D, cap, scale):
    """Ordinary scores (products of q and k are as small as the scale is large) far below the cap, which takes nothing away"""
    q, k, v = normal((3, 1, 2, 150, D), 4)
    q, k = q * (scale ** -0.5 / 4), k * (scale ** -0.5 / 4)
    d = np.stack([documents(150, (100, 50))])
    got = attend(q, k, v, torch.from_numpy(d).cuda(), cap=cap, scale=scale)
    o, p = po.attention(widen(q), widen(k), widen(v), d, None, cap, scale)
    assert_within(got, o, bound(widen(q), widen(k), widen(v), p, o, 0.0, scale, po.visible(d)))


@pytest.mark.parametrize("cap,scale", [(1e14, 1e17), (1e35, 3e38), (1e5, 1e9), (1e30, 1e32), (1e-20, 1e-17)], ids=str)
def test_products_of_zero_under_any_cap(cap, scale):
    q, k, v = normal((3, 1, 2, 100, 64), 4)
    got = attend(q * 0, k, v, torch.zeros(100, dtype=torch.int32, device="cuda"), cap=cap, scale=scale)
    want, size = (np.broadcast_to(t.mean(2, keepdims=True), t.shape) for t in (widen(v), np.abs(widen(v))))
    assert_within(got, want, BF16_STEP * np.abs(want) + 102 * 2.0 ** -23 * size)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("to,cap", [(2.0 ** 110, 0.5), (2.0 ** 119, 2.0 ** -20), (2.0 ** 100, 1.0)], ids=str)
def test_scales_far_above_the_cap(D, to, cap):
    """Products of q and k of 2^-98 or so under a scale that takes them beyond the cap: every score is the cap or its negative"""
    q, k, v = normal((3, 1, 2, 150, D), 4)
    k = (torch.where(k[..., :1] > 0, 1.0, -1.0) * 2.0 ** -52).expand_as(k).contiguous().to(k.dtype)
    q = torch.ones_like(q) * 2.0 ** -52
    d = np.stack([documents(150, (100, 50))])
    got = attend(q, k, v, torch.from_numpy(d).cuda(), cap=cap, scale=to)
    o, p = po.attention(widen(q), widen(k), widen(v), d, None, cap, to)
    assert_within(got, o, bound(0 * widen(q), widen(k), widen(v), p, o, cap, to, po.visible(d)))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap,scale", [(3e38, 1e35), (1e38, 1e35), (5e37, 1e35), (3e38, 0.0)], ids=str)
def test_caps_near_the_largest_number(D, cap, scale):
    """Ordinary scores stay what they are under them"""
    q, k, v = normal((3, 1, 2, 150, D), 4)
    s = scale if scale else D ** -0.5
    if scale:
        q, k = q * (scale ** -0.5 / 4), k * (scale ** -0.5 / 4)
    d = np.stack([documents(150, (100, 50))])
    got = attend(q, k, v, torch.from_numpy(d).cuda(), cap=cap, scale=scale)
    o, p = po.attention(widen(q), widen(k), widen(v), d, None, cap, s)
    assert_within(got, o, bound(widen(q), widen(k), widen(v), p, o, 0.0, s, po.visible(d)))


@pytest.mark.parametrize("kw", [dict(cap=1e-46), dict(cap=1e-300), dict(scale=1e-46), dict(cap=2.0, scale=5e-324)], ids=str)
def test_caps_and_scales_that_fp32_holds_as_zero(form, kw):  # noqa: F811
    """They would be taken for no cap and for the usual scale"""
    q, k, v = normal((3, 1, 2, 100, 64), 4)
    o = torch.full_like(q, 7.0)
    with pytest.raises(ValueError):
        attend(q, k, v, torch.zeros(100, dtype=torch.int32, device="cuda"), o=o, **kw)
    assert (o == 7.0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [94, -100])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_values_far_from_one(D, power, cap):
    """|V| up to 2^97 cannot overflow, whatever the scores: of keys whose scores climb a weight is 2^8 at most against its row's reference"""
    N, lengths = 700, (400, 250)
    q, k, v = normal((3, 1, 1, N, D), 4)
    k = torch.linspace(-0.6, 0.6, N, device="cuda")[:, None].expand_as(k) + 0.05 * k.float()
    q, k, v = q * 0 + 2.0, k.to(q.dtype), v * 2.0 ** power
    d = np.stack([documents(N, lengths)])
    got = attend(q, k, v, torch.from_numpy(d).cuda(), cap=cap)
    o, p = po.attention(widen(q), widen(k), widen(v), d, None, cap)
    assert_within(got, o, bound(widen(q), widen(k), widen(v), p, o, cap, D ** -0.5, po.visible(d)))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where", ["k", "v", "both"])
@pytest.mark.parametrize("value", [NAN, float("inf"), -float("inf"), 3.3895e38])
def test_what_is_not_visible_has_no_part_under_a_cap(D, where, value):
    """As without one: infinities and NaN in padding, in other documents and in tokens of a later order, in tiles that others share"""
    N, bad = 250, [95, 129, 229, 240, 249]
    d, order = documents(N, (90, 40, 100)), np.arange(N, dtype=np.int32) // 10
    q, k, v = normal((3, 1, 2, N, D), 5)
    q *= 3.0
    clean = [widen(t) for t in (q, k, v)]
    for t in (k, v):
        if where in ("both", "k" if t is k else "v"):
            t[:, :, bad, 3:9] = value
    got = widen(attend(q, k, v, torch.from_numpy(d).cuda(), torch.from_numpy(order).cuda(), 10.0))
    see = po.visible(d[None], order[None])
    fine = ~see[0][:, bad].any(1)
    assert fine[:90].all() and fine.sum() > 150
    o, p = po.attention(*clean, d[None], order[None], 10.0)
    off = bound(*clean, p, o, 10.0, D ** -0.5, see)
    assert (np.abs(got - o) <= off)[:, :, fine].all()
    if where == "v" and not np.isfinite(value):
        assert not np.isfinite(got[:, :, ~fine & (d >= 0)][..., 3:9]).any() and np.isfinite(got[:, :, ~fine][..., 9:]).all()
