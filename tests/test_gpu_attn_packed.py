"""rapid_attn_packed against the fp64 oracle."""
import numpy as np
import pytest
import torch

import paper_2509_22323_amd as ra
from layer_common import BF16_STEP, NAN, normal, widen
from oracle import packed_oracle as po

pytestmark = pytest.mark.gpu


def documents(N, lengths, seed=None):
    """[N]: the documents one after the other, or, with a seed, their tokens mixed; -1 behind"""
    d = np.concatenate([np.full(n, i) for i, n in enumerate(lengths)] + [np.full(N - sum(lengths), -1)])
    return (d if seed is None else np.random.default_rng(seed).permutation(d)).astype(np.int32)


def bound(q, k, v, p, o, cap, scale, see):
    """What rounding can do to an output o = sum p v, p the softmax.  A weight is rounded to bf16 (2^-8, half a step), and its exponent is off
    by what the score's D products and their sums round to (2^-23 of their absolute values a time, whichever way the matrix unit
    rounds), by the few roundings of the exponent itself (2^-21 of the largest, and cap: those of tanh, 2^-20 of the cap) and by what
    exp2 is off (2^-22).  Numerator and sum take the same rounded weights, so what is off by e relative in each of them moves o by e
    sum p |v - o| at most; sums over the keys round by 2^-23 of their absolute values a time; then half a step of bf16."""
    D, N = q.shape[-1], k.shape[-2]
    size = np.matmul(np.abs(q), np.swapaxes(np.abs(k), -1, -2)) * scale
    size = np.where(see[:, None], size, 0.0).max(-1, keepdims=True)
    e = BF16_STEP + (D + 1) * 2.0 ** -23 * size + 2.0 ** -20 * (cap + np.minimum(size, cap if cap else np.inf)) + 2.0 ** -21
    spread = np.stack([np.stack([(p[b, h][..., None] * np.abs(v[b, h][None] - o[b, h][:, None])).sum(1) for h in range(q.shape[1])]) for b in range(q.shape[0])])
    off = e * (1 + 2 * e) * spread + (N + 2) * 2.0 ** -22 * np.matmul(p, np.abs(v))
    return off + BF16_STEP * (np.abs(o) + off) + 2.0 ** -134


def check(B, H, D, n, m, document, order=None, cap=0.0, scale=0.0, spread=1.0, seed=1, fused=True, shared=False):
    """n and m tokens in two segments (m = 0: one); document, order [N] or [B, N]."""
    segments, big = [], []
    for i, t in enumerate((n, m)):
        if t == 0:
            continue
        if fused:
            q, k, v = normal((B, t, 3, H, D), seed + i).permute(2, 0, 3, 1, 4)
            o = torch.full((B, t, H, D), NAN, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        else:                                          # head after head, in the middle of more tokens
            q, k, v = normal((3, B, H, t + 5, D), seed + i)[..., 2:2 + t, :]
            o = torch.full((B, H, t + 3, D + 8), NAN, dtype=torch.bfloat16, device="cuda")
            big.append((o, t))
            o = o[:, :, 1:1 + t, :D]
        q.mul_(spread)
        segments.append((q, k, v, o))
    document = np.broadcast_to(np.asarray(document, np.int32), (B, n + m))
    order = None if order is None else np.broadcast_to(np.asarray(order, np.int32), (B, n + m))
    dt, ot = (None if a is None else torch.from_numpy(np.array(a[0] if shared else a)).cuda() for a in (document, order))
    got = ra.rapid_attn_packed(segments, dt, ot, cap=cap, scale=scale)
    assert all(a is s[3] for a, s in zip(got, segments))
    q, k, v = (np.concatenate([widen(s[i]) for s in segments], 2) for i in range(3))
    s = scale if scale > 0 else D ** -0.5
    o, p = po.attention(q, k, v, document, order, cap, s)
    e = bound(q, k, v, p, o, cap, s, po.visible(document, order))
    out = np.concatenate([widen(t) for t in got], 2)
    assert np.isfinite(out).all()
    over = np.abs(out - o) - e
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, f"{out[at]} for {o[at]} at {at}, bound {e[at]:.3e}; {(over > 0).sum()} of {over.size} beyond"
    none = np.broadcast_to((document < 0)[:, None, :, None], out.shape)
    assert not out[none].any()
    for buffer, t in big:
        assert torch.isnan(buffer[:, :, 0]).all() and torch.isnan(buffer[:, :, 1 + t:]).all() and torch.isnan(buffer[..., D:]).all()
    return got


SIZES = [(1, 0, (1,)), (1, 1, (1, 1)), (2, 0, (1, 1)), (15, 2, (17,)), (16, 0, (5, 11)), (31, 33, (64,)), (64, 0, (64,)), (65, 0, (1, 63, 1)), (63, 65, (40, 88)),
         (127, 1, (128,)), (128, 128, (100, 156)), (129, 0, (129,)), (100, 77, (3, 100, 1, 60)), (192, 64, (256,)), (257, 31, (200, 20, 60)), (300, 100, (7,) * 50),
         (512, 0, (300, 212)), (333, 200, (533,)), (640, 77, (500, 217))]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,m,lengths", SIZES, ids=str)
def test_documents_one_after_the_other(D, n, m, lengths):
    check(1, 2, D, n, m, documents(n + m, lengths), seed=n + m)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("fused", [False, True])
def test_documents_over_both_segments(D, cap, fused):
    """Images, then texts, then padding; two samples of different documents"""
    images, texts = (130, 64, 1, 60), (20, 1, 33, 7)
    d = np.stack([np.concatenate([documents(255, images), documents(70, texts)]), np.concatenate([documents(255, images[::-1]), documents(70, texts[::-1])])])
    check(2, 3, D, 255, 70, d, cap=cap, spread=4.0 if cap else 1.0, fused=fused)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,m,lengths", [(100, 30, (40, 1, 60)), (256, 0, (100, 100)), (400, 113, (200, 200, 50, 1, 60))], ids=str)
def test_documents_in_any_order(D, n, m, lengths):
    check(2, 2, D, n, m, np.stack([documents(n + m, lengths, 3), documents(n + m, lengths[::-1], 4)]) * 1000 - (np.arange(n + m) < 0), seed=7)


def test_document_numbers_are_any():
    """The largest, and those whose distance is no 32-bit number"""
    d = np.concatenate([np.full(70, 2 ** 31 - 1), np.full(50, 0), np.full(30, -(2 ** 31)), np.full(60, 2 ** 31 - 2), np.full(45, -1)])
    check(1, 2, 64, 255, 0, d)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 10.0])
@pytest.mark.parametrize("kind", ["causal", "prefix", "text_first", "frames", "any", "reversed"])
def test_orders(D, cap, kind):
    n, m, lengths = 300, 81, (150, 1, 200, 20)
    N = n + m
    d = documents(N, lengths)
    at = np.concatenate([np.arange(k) for k in lengths] + [np.zeros(N - sum(lengths), int)])
    order = {"causal": at, "prefix": np.maximum(at - 30, 0), "text_first": np.arange(N) < n, "frames": at // 37,
             "any": np.random.default_rng(2).integers(-2 ** 31, 2 ** 31 - 1, N), "reversed": -np.arange(N)}[kind]
    check(1, 2, D, n, m, d, order, cap=cap, spread=3.0 if cap else 1.0)


def test_one_document_and_one_order_for_all_samples():
    check(3, 1, 64, 200, 0, documents(200, (90, 100)), np.arange(200), shared=True)
    check(3, 2, 128, 130, 40, documents(170, (170,)), shared=True)


@pytest.mark.parametrize("cap", [0.5, 5.0, 30.0, 50.0, 300.0, 1e30])
@pytest.mark.parametrize("spread", [0.01, 1.0, 8.0])
def test_caps(cap, spread):
    """Scores far below their cap, at it and beyond"""
    for D in (64, 128):
        check(1, 2, D, 200, 0, documents(200, (120, 80)), cap=cap, spread=spread)


@pytest.mark.parametrize("spread", [4.0, 16.0])
@pytest.mark.parametrize("D", [64, 128])
def test_peaked_rows(D, spread):
    check(1, 2, D, 400, 50, documents(450, (250, 200)), spread=spread)


@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_climb(D):
    """Every key's score is far above those before it: the reference of the exponents moves all the way"""
    n = 320
    q, k, v = normal((3, 1, 1, n, D), 3)
    k.copy_((torch.linspace(-30, 30, n, device="cuda")[:, None] * torch.ones(D, device="cuda")).to(torch.bfloat16)[None, None])
    q.fill_(1.0)
    o = torch.empty_like(q)
    for turn in (k, k.flip(2).contiguous()):
        ra.rapid_attn_packed([(q, turn, v, o)], torch.zeros(n, dtype=torch.int32, device="cuda"))
        want, p = po.attention(widen(q), widen(turn), widen(v), np.zeros((1, n), int))
        assert np.abs(widen(o) - want).max() <= 2.0 ** -6 * np.abs(want).max()


def test_scales():
    check(1, 1, 64, 150, 0, documents(150, (150,)), scale=0.5)
    check(1, 1, 128, 150, 0, documents(150, (150,)), scale=1e-3)
    check(1, 1, 128, 150, 0, documents(150, (150,)), scale=0.3, cap=2.0)


@pytest.mark.parametrize("D", [64, 128])
def test_no_document_at_all(D):
    q, k, v = normal((3, 1, 2, 200, D), 3)
    o = torch.full_like(q, NAN)
    ra.rapid_attn_packed([(q, k, v, o)], torch.full((200,), -1, dtype=torch.int32, device="cuda"))
    assert not o.any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where", ["k", "v", "both"])
@pytest.mark.parametrize("value", [NAN, float("inf"), -float("inf"), 3.3895e38])
def test_what_is_not_visible_has_no_part(D, where, value):
    """Infinities and NaN in padding, in other documents and in tokens of a later order, in tiles that others share"""
    n, m, lengths = 200, 50, (90, 40, 100)
    N = n + m
    d = documents(N, lengths)
    order = np.arange(N) // 10
    q, k, v = normal((3, 1, 2, N, D), 5)
    ot, dt = torch.from_numpy(order.astype(np.int32)).cuda(), torch.from_numpy(d).cuda()

    def run():
        o = torch.full((1, 2, N, D), 7.0, dtype=torch.bfloat16, device="cuda")
        segments = [tuple(t[:, :, a:z] for t in (q, k, v, o)) for a, z in ((0, n), (n, N))]
        ra.rapid_attn_packed(segments, dt, ot)
        return o

    want = run()
    bad = [95, 129, 229, 240, 249]                     # in the second and third document and in padding
    for t in (k, v):
        if where in ("both", "k" if t is k else "v"):
            t[:, :, bad, 3:9] = value
    got = run()
    see = po.visible(d[None], order[None])[0]
    fine = torch.from_numpy(~see[:, bad].any(1)).cuda()
    assert fine[:90].all() and fine.sum() > 150
    assert torch.equal(got[:, :, fine].view(torch.int16), want[:, :, fine].view(torch.int16)) or \
        (got[:, :, fine].double() - want[:, :, fine].double()).abs().max() <= 2.0 ** -6
    if where == "v" and not np.isfinite(value):
        hit = torch.from_numpy(see[:, bad].any(1)).cuda()
        assert not torch.isfinite(got[:, :, hit][..., 3:9].float()).any()
        assert torch.isfinite(got[:, :, hit][..., 9:].float()).all()


def test_a_request_packed_is_the_request_alone():
    """Within the rounding of weights, whatever it is packed with"""
    D, H = 128, 2
    alone = normal((3, 1, H, 150, D), 1)
    others = normal((3, 1, H, 700, D), 2)
    want = torch.empty_like(alone[0])
    ra.rapid_attn_packed([(*alone, want)], torch.zeros(150, dtype=torch.int32, device="cuda"))
    for at in (0, 1, 63, 64, 500):
        q, k, v = (torch.cat([o[:, :, :at], a, o[:, :, at:]], 2) for o, a in zip(others, alone))
        d = torch.full((850,), 3, dtype=torch.int32, device="cuda")
        d[at:at + 150] = 9
        o = torch.empty_like(q)
        ra.rapid_attn_packed([(q, k, v, o)], d)
        assert (o[:, :, at:at + 150].double() - want.double()).abs().max() <= 2.0 ** -6


def test_it_is_the_dense_attention_where_there_is_one_document():
    q, k, v = normal((3, 2, 3, 512, 128), 1)
    a, b = torch.empty_like(q), torch.empty_like(q)
    ra.rapid_attn_dense(q, k, v, a)
    ra.rapid_attn_packed([(q, k, v, b)], torch.zeros(512, dtype=torch.int32, device="cuda"))
    assert (a.double() - b.double()).abs().max() <= 2.0 ** -7


@pytest.mark.parametrize("D", [64, 128])
def test_heads_and_samples(D):
    check(3, 5, D, 70, 0, np.stack([documents(70, (30, 30)), documents(70, (70,)), documents(70, (1,))]))
    check(1, 70, D, 40, 8, documents(48, (20, 28)))


def test_longer_sequences_at_some_rows():
    """9000 tokens of four documents, a prefix order: rows of every document against the oracle"""
    H, D, lengths = 2, 128, (5000, 2500, 1000, 300)
    N = 9000
    d = documents(N, lengths)
    at = np.concatenate([np.arange(k) for k in lengths] + [np.zeros(N - sum(lengths), int)])
    for order, cap in ((None, 0.0), (np.maximum(at - 700, 0).astype(np.int32), 20.0)):
        q, k, v = normal((3, 1, H, N, D), 1)
        o = torch.full_like(q, NAN)
        ra.rapid_attn_packed([(q, k, v, o)], torch.from_numpy(d).cuda(), None if order is None else torch.from_numpy(order).cuda(), cap=cap)
        rows = np.concatenate([np.random.default_rng(1).integers(0, 8800, 40), [0, 4999, 5000, 7499, 7500, 8499, 8500, 8799]])
        see = po.visible(d[None], None if order is None else order[None])[0][rows]
        s = np.matmul(widen(q)[0][:, rows], np.swapaxes(widen(k)[0], 1, 2)) * D ** -0.5
        s = np.where(see, cap * np.tanh(s / cap) if cap else s, -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        want = np.matmul(p, widen(v)[0]) / p.sum(-1, keepdims=True)
        got = widen(o)[0]
        # weights off by 2^-8 at random and by the exponent's part; the largest of 12288 outputs
        assert np.abs(got[:, rows] - want).max() <= 2.0 ** -7 * np.sqrt((p ** 2).sum(-1) / p.sum(-1) ** 2).max() * 4 + BF16_STEP * np.abs(want).max()
        assert not got[:, 8800:].any() and np.isfinite(got).all()


def test_two_streams_at_once():
    cases, want = [], []
    for seed in range(2):
        q, k, v = normal((3, 1, 4, 700, 64), seed)
        d = torch.from_numpy(documents(700, (300, 200, 100))).cuda()
        cases.append((q, k, v, torch.empty_like(q), d))
        want.append(ra.rapid_attn_packed([(q, k, v, torch.empty_like(q))], d)[0].clone())
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for (q, k, v, o, d), s in zip(cases, streams):
            with torch.cuda.stream(s):
                ra.rapid_attn_packed([(q, k, v, o)], d)
    torch.cuda.synchronize()
    for (_, _, _, o, _), w in zip(cases, want):
        assert torch.equal(o.view(torch.int16), w.view(torch.int16))
