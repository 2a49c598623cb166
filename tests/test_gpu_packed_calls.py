"""Calls of the operators over packed sequences that their documentation allows or excludes, in both forms of the binding."""
import numpy as np
import pytest
import torch

import paper_2509_22323_amd as ra
from layer_common import BF16_STEP, NAN, assert_within, normal, widen
from oracle import packed_oracle as po
from test_gpu_attn_packed import bound, check, documents
from test_gpu_int8 import codes, scales

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "python"])
def form(request, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(ra.binding, "_native", ra.binding._NoNative())
    return request.param


def attend(q, k, v, d, order=None, cap=0.0, scale=0.0, o=None, own=True):
    B, H, N, D = q.shape
    workspace = torch.empty(ra.rapid_attn_packed_workspace_bytes(B, H, N, D), dtype=torch.uint8, device="cuda") if own else None
    return ra.rapid_attn_packed([(q, k, v, torch.full_like(q, NAN) if o is None else o)], d, order, cap, scale, workspace)[0]


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def test_both_forms_give_the_same_bits(monkeypatch):
    x, w, b, g = normal((2, 70, 128), 1), normal((96, 128), 2), normal((96,), 3), normal((3, 96), 4)
    d = torch.from_numpy(np.random.default_rng(1).integers(-1, 3, (2, 70)).astype(np.int32)).cuda()
    s, t = normal((3, 128), 5), normal((3, 128), 6)
    q, k, v = normal((3, 2, 3, 300, 64), 7)
    dt = torch.from_numpy(documents(300, (100, 150))).cuda()

    def run():
        empty = lambda *shape: torch.zeros(shape, dtype=torch.int8, device="cuda")
        wq, ws = ra.rapid_quantize_rows(w, empty(96, 128), torch.zeros(96, device="cuda"))
        xq, xs = ra.rapid_norm_modulate_int8(x, empty(2, 70, 128), torch.zeros(2, 70, device="cuda"), s, t, 1e-5, d)
        y = ra.rapid_linear_int8(xq, xs, wq, ws, torch.zeros(2, 70, 96, dtype=x.dtype, device="cuda"), b, "silu", g, None, d)
        return [wq, ws, xq, xs, y, attend(q, k, v, dt), attend(q, k, v, dt, dt * 0 + torch.arange(300, device="cuda", dtype=torch.int32), 4.0, 0.2)]

    native = run()
    monkeypatch.setattr(ra.binding, "_native", ra.binding._NoNative())
    assert all(same(a, b) for a, b in zip(native, run()))


def test_tensors_that_require_gradients_are_taken_and_nothing_is_recorded(form):
    x, w, q = normal((1, 9, 64), 1), normal((40, 64), 2), normal((1, 2, 9, 64), 3)
    d = torch.zeros(9, dtype=torch.int32, device="cuda")

    def calls(x, w, q):
        empty = lambda *shape: torch.zeros(shape, dtype=torch.int8, device="cuda")
        wq, ws = ra.rapid_quantize_rows(w, empty(40, 64), torch.zeros(40, device="cuda"))
        xq, xs = ra.rapid_norm_modulate_int8(x, empty(1, 9, 64), torch.zeros(1, 9, device="cuda"))
        return [wq, ws, xq, xs, ra.rapid_linear_int8(xq, xs, wq, ws, torch.zeros(1, 9, 40, dtype=x.dtype, device="cuda"), residual=None),
                attend(q, q + 0, q * 2, d, o=torch.zeros(1, 2, 9, 64, dtype=q.dtype, device="cuda"))]

    want = calls(x, w, q)
    for a, b in zip(calls(*(t.clone().requires_grad_() for t in (x, w, q))), want):
        assert a.grad_fn is None and not a.requires_grad and same(a, b)


FAR = (1 << 32) + 1                                        # 1 in its low 32 bits


def test_sizes_beyond_32_bits(form):
    """(one element for each row, so that nothing is allocated)"""
    x, x8, w8, y = normal((1, 64), 1), codes((1, 64), 1), codes((40, 64), 2), torch.zeros(1, 40, dtype=torch.bfloat16, device="cuda")
    one, forty, q = torch.ones(1, device="cuda"), torch.ones(40, device="cuda"), normal((1, 1, 1, 64), 3)
    d, ws = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(4096, dtype=torch.uint8, device="cuda")
    kept = [t.clone() for t in (x, x8, y, q)]
    calls = [lambda: ra.rapid_quantize_rows(x.expand(FAR, 64), x8.expand(FAR, 64), one.expand(FAR)), lambda: ra.rapid_norm_modulate_int8(x.expand(FAR, 64), x8.expand(FAR, 64), one.expand(FAR)),
             lambda: ra.rapid_linear_int8(x8.expand(FAR, 64), one.expand(FAR), w8, forty, y.expand(FAR, 40)),
             lambda: ra.rapid_linear_int8(x8, one, w8[:1].expand(FAR, 64), one.expand(FAR), y[:, :1].expand(1, FAR))]
    for shape in ((FAR, 1, 1, 64), (1, FAR, 1, 64), (1, 1, FAR, 64)):
        calls.append(lambda s=shape: ra.rapid_attn_packed([(q.expand(s), q.expand(s), q.expand(s), q.clone().expand(s))], d, workspace=ws))
    for call in calls:
        with pytest.raises((ra.RapidAttnError, TypeError, ValueError)):
            call()
    assert all(torch.equal(a, b) for a, b in zip((x, x8, y, q), kept))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [350.0, 1e4, 1e6, 1e12, 1e30, 3.4e38])
def test_caps_far_above_the_scores(D, cap):
    """Such a cap takes nothing away: what scores round to is in proportion to them, not to the cap"""
    q, k, v = normal((3, 1, 2, 150, D), 4)
    d = np.stack([documents(150, (100, 50))])
    for spread in (1.0, 8.0):
        got = attend(q * spread, k, v, torch.from_numpy(d).cuda(), cap=cap)
        o, p = po.attention(widen(q * spread), widen(k), widen(v), d, None, cap)
        assert_within(got, o, bound(widen(q * spread), widen(k), widen(v), p, o, 0.0, D ** -0.5, po.visible(d)))


@pytest.mark.parametrize("D", [64, 128])
def test_caps_between_small_and_large_scores(D):
    """Tiles that hold scores far below the cap and others at it: rows of small queries as if they were alone"""
    q, k, v = normal((3, 1, 2, 200, D), 4)
    q[:, :, ::2] *= 0.02
    q[:, :, 1::2] *= 100.0
    d = np.zeros((1, 200), np.int32)
    for cap in (20.0, 300.0, 2000.0):
        got = attend(q, k, v, torch.from_numpy(d).cuda(), cap=cap)[:, :, ::2]
        o, p = half(q, k, v, cap)
        assert_within(got, o, bound(widen(q[:, :, ::2]), widen(k), widen(v), p, o, 0.0, D ** -0.5, np.ones((1, 100, 200), bool)))


def half(q, k, v, cap):
    """Output and softmax of every second query over all keys"""
    s = np.matmul(widen(q[:, :, ::2]), np.swapaxes(widen(k), -1, -2)) * q.shape[-1] ** -0.5
    p = np.exp(cap * np.tanh(s / cap))
    p /= p.sum(-1, keepdims=True)
    return np.matmul(p, widen(v)), p


@pytest.mark.parametrize("cap,scale", [(0.0, 3e38), (0.0, 1e-44), (1e-44, 0.0), (1e-30, 3e38), (3e38, 1e-44), (3e38, 3e38)], ids=str)
def test_caps_and_scales_at_the_ends_of_fp32(cap, scale):
    """Products of 0 have the exponent 0 under all of them"""
    q, k, v = normal((3, 1, 2, 100, 64), 4)
    d = documents(100, (60, 40))
    got = attend(q * 0, k, v, torch.from_numpy(d).cuda(), cap=cap, scale=scale)
    for a, z in ((0, 60), (60, 100)):
        mean = widen(v)[:, :, a:z].mean(2, keepdims=True)
        size = np.abs(widen(v)[:, :, a:z]).mean(2, keepdims=True)
        want = np.broadcast_to(mean, (1, 2, z - a, 64))
        assert_within(got[:, :, a:z], want, BF16_STEP * np.abs(want) + 2.0 ** -15 * size)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 4.0])
def test_few_groups_of_many_tiles(D, cap):
    """Tiles of a group that several workgroups share, over two segments: in turn, in any order, and rows that see nothing of a share"""
    N, lengths = 1160, (500, 300, 1, 300)
    for d, order in ((documents(N, lengths), None), (documents(N, lengths, 3), np.arange(N) % 97), (documents(N, (64, 1000)), np.arange(N))):
        check(1, 1, D, 703, N - 703, d, order, cap=cap, spread=3.0 if cap else 1.0)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N", [700, 1500])
@pytest.mark.parametrize("value", [NAN, float("inf"), -float("inf")])
def test_shares_of_tiles_that_hold_what_is_not_visible(D, N, value):
    q, k, v = normal((3, 1, 1, N, D), 5)
    d = documents(N, (N // 2, N // 3))
    want = attend(q, k, v, torch.from_numpy(d).cuda())
    bad = [N // 2 + 3, N - 5]
    for t in (k, v):
        t[:, :, bad, 3:9] = value
    got = attend(q, k, v, torch.from_numpy(d).cuda())
    a = N // 2
    # (a row that has taken an infinity into a sum is summed again, in another order: weights off by half a step of bf16 each)
    _, p = po.attention(widen(q[:, :, :a]), widen(k[:, :, :a]), widen(v[:, :, :a]), d[None, :a])
    off = 2 * BF16_STEP * np.matmul(p, np.abs(widen(v[:, :, :a]))) + 2 * BF16_STEP * np.abs(widen(want[:, :, :a]))
    assert_within(got[:, :, :a], widen(want[:, :, :a]), off)
    assert not torch.isfinite(got[:, :, a:a + N // 3, 3:9].float()).any() and not got[:, :, a + N // 3:].any()


def rows_of(q, k, v, d, order, cap, rows):
    see = po.visible(d[None], None if order is None else order[None]) if len(d) < 20000 else None
    out = []
    for r in rows:
        keys = (d == d[r]) & ((order <= order[r]) if order is not None else True) if see is None else see[0, r]
        s = np.einsum("hd,hkd->hk", widen(q[0, :, r]), widen(k[0])[:, keys]) * q.shape[-1] ** -0.5
        s = cap * np.tanh(s / cap) if cap else s
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        vk = widen(v[0])[:, keys]
        o = np.einsum("hk,hkd->hd", p, vk)
        # weights off by half a step of bf16 and the exponents' 2^-10 (D products of at most 8 each, see the other tests), sums in fp32
        e = BF16_STEP + 2.0 ** -10
        out.append((o, e * np.einsum("hk,hkd->hd", p, np.abs(vk - o[:, None])) + (len(d) + 2) * 2.0 ** -22 * np.einsum("hk,hkd->hd", p, np.abs(vk)) + BF16_STEP * np.abs(o)))
    return np.stack([o for o, _ in out], 1), np.stack([e for _, e in out], 1)


@pytest.mark.parametrize("order", [False, True])
def test_seventy_thousand_tokens(order):
    """(more tiles than are put in order, or listed at a time)"""
    N, D = 70003, 64
    q, k, v = normal((3, 1, 1, N, D), 1)
    d = documents(N, (40000, 1, 20000, 9000))
    at = np.arange(N).astype(np.int32) if order else None
    got = attend(q, k, v, torch.from_numpy(d).cuda(), torch.from_numpy(at).cuda() if order else None)
    rows = [0, 1, 777, 39999, 40000, 40001, 50000, 60000, 60001, 69000]
    want, e = rows_of(q, k, v, d, at, 0.0, rows)
    assert_within(got[0][:, rows], want, e)
    assert torch.isfinite(got.float()).all() and not got[:, :, 69001:].any()


def test_heads_and_rows_beyond_32_bits():
    """Rows and heads whose offsets are no 32-bit numbers, the largest stride of a row"""
    far, n = (1 << 23) - 8, 270
    store = torch.empty(far * n + 512, dtype=torch.bfloat16, device="cuda")
    q, k, v, o = (store.as_strided((1, 1, n, 64), (0, 0, far, 1), 64 * i) for i in range(4))
    for t, seed in ((q, 1), (k, 2), (v, 3)):
        t.copy_(normal((1, 1, n, 64), seed))
    d = torch.from_numpy(documents(n, (200, 60))).cuda()
    near = [t.clone() for t in (q, k, v)]
    attend(q, k, v, d, o=o)
    assert same(o, attend(*near, d))
    heads = [store.as_strided((1, 2, n, 64), (0, (1 << 31) + 64, 64, 1), 64 * n * i) for i in range(4)]
    near = [normal((1, 2, n, 64), seed) for seed in (4, 5, 6)]
    for a, b in zip(heads, near):
        a.copy_(b)
    attend(*heads[:3], d, o=heads[3])
    assert same(heads[3], attend(*near, d))


def test_segments_of_different_strides():
    n, m, D, H = 100, 90, 64, 3
    whole = normal((3, 1, H, n + m, D), 2)
    d = torch.from_numpy(documents(n + m, (50, 90, 30))).cuda()
    want = attend(*whole, d)
    first = [t[:, :, :n].clone() for t in whole]                                    # head after head
    second = whole[:, :, :, n:].permute(1, 3, 0, 2, 4).contiguous().permute(2, 0, 3, 1, 4)       # token after token, q, k, v side by side
    o = torch.empty(1, n, H, D, dtype=torch.bfloat16, device="cuda").transpose(1, 2), torch.empty(1, H, m, D, dtype=torch.bfloat16, device="cuda")
    ra.rapid_attn_packed([(*first, o[0]), (*second, o[1])], d)
    # (tiles are counted within a segment, so sums are in another order)
    _, p = po.attention(*(widen(t) for t in whole), d.cpu().numpy()[None])
    assert_within(torch.cat(o, 2), widen(want), 2 * BF16_STEP * (np.matmul(p, np.abs(widen(whole[2]))) + np.abs(widen(want))))


@pytest.mark.parametrize("N,H", [(200, 2), (1300, 2), (4200, 24)], ids=str)
def test_a_captured_call(N, H):
    """Replayed over other inputs and documents, with eager calls in between, on workspaces of its own"""
    D = 64
    q, k, v = normal((3, 1, H, N, D), 1)
    o, cut = torch.empty_like(q), N // 3
    d = torch.from_numpy(documents(N, (cut, N // 2))).cuda()
    ws = torch.empty(ra.rapid_attn_packed_workspace_bytes(1, H, N, D), dtype=torch.uint8, device="cuda")
    call = lambda out, space: ra.rapid_attn_packed([(q, k, v, out)], d, cap=3.0, workspace=space)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call(o, ws)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(o, ws)
    for i in range(4):
        q.copy_(normal(q.shape, 10 + i))
        d.copy_(torch.from_numpy(documents(N, (cut - 7 * i, N // 2 - 100 + 20 * i), seed=i if i == 3 else None)).cuda())
        want = call(torch.empty_like(q), None)[0]
        o.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert same(o, want), i


def test_two_graphs_on_two_streams():
    graphs, outs, wants = [], [], []
    for seed in range(2):
        q, k, v = normal((3, 1, 2, 1300, 128), seed)
        d = torch.from_numpy(documents(1300, (900, 300))).cuda()
        o, ws = torch.empty_like(q), torch.empty(ra.rapid_attn_packed_workspace_bytes(1, 2, 1300, 128), dtype=torch.uint8, device="cuda")
        wants.append(attend(q, k, v, d).clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ra.rapid_attn_packed([(q, k, v, o)], d, workspace=ws)
        graphs.append((graph, q, k, v, d, ws))
        outs.append(o)
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (graph, *_) in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(outs, wants))


def test_a_captured_product_with_a_workspace():
    """(pieces of a long axis, joined: the second launch is part of the graph)"""
    x, w, xs, ws = codes((1, 60, 8192), 1), codes((512, 8192), 2), scales((1, 60), 3, 0.01), scales((512,), 4, 0.01)
    need = ra.rapid_linear_int8_workspace_bytes(60, 512, 8192)
    space = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    o = torch.empty(1, 60, 512, dtype=torch.bfloat16, device="cuda")
    run = lambda out, space: ra.rapid_linear_int8(x, xs, w, ws, out, workspace=space)
    run(o, space)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(o, space)
    for i in range(4):
        x.copy_(codes((1, 60, 8192), 10 + i))
        want = run(torch.empty_like(o), None)
        o.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert same(o, want), i


def test_many_samples_and_heads():
    """More pairs than a multiple of 8, one token each"""
    q, k, v = normal((3, 31, 33, 1, 64), 1)
    d = torch.zeros(31, 1, dtype=torch.int32, device="cuda")
    d[5] = -1
    got = attend(q, k, v, d)
    want = v.clone()
    want[5] = 0
    assert same(got, want)


@pytest.mark.parametrize("C", [2056, 2432, 2816, 4104, 4608, 6144, 8200, 9728, 12288, 12296])
def test_norms_of_every_width(C):
    from test_gpu_int8 import assert_normed
    x = normal((1, 7, C), C, 2.0, 0.5)
    s, t = normal((1, C), 1), normal((1, C), 2)
    q, scale = torch.zeros((1, 7, C), dtype=torch.int8, device="cuda"), torch.zeros((1, 7), device="cuda")
    ra.rapid_norm_modulate_int8(x, q, scale, s, t, 1e-6)
    assert_normed(po.norm_modulate(widen(x), widen(s), widen(t), float(np.float32(1e-6))), (q, scale))


@pytest.mark.parametrize("parts", [dict(), dict(bias=True), dict(gate=True), dict(residual=True), dict(bias=True, residual=True), dict(bias=True, gate=True, residual=True),
                                   dict(gate=True, residual=True, document=True), dict(bias=True, act="silu", residual=True, document=True)], ids=str)
@pytest.mark.parametrize("K,N,M", [(1552, 300, 2000), (144, 1000, 5000), (2432, 2432, 1100)], ids=str)
def test_a_row_gives_the_same_bits_under_every_epilogue(parts, K, N, M):
    x, w, xs, ws = codes((1, M, K), 1), codes((N, K), 2), scales((1, M), 3, 0.01), scales((N,), 4, 0.01)
    d = torch.zeros((1, M), dtype=torch.int32, device="cuda") if parts.get("document") else None
    b = normal((N,), 5) if parts.get("bias") else None
    g = normal((1, N), 6) if parts.get("gate") else None
    r = normal((1, M, N), 7, 30.0) if parts.get("residual") else None

    def run(a, z):
        return ra.rapid_linear_int8(x[:, a:z], xs[:, a:z].contiguous(), w, ws, torch.empty((1, z - a, N), dtype=torch.bfloat16, device="cuda"), b,
                                    parts.get("act", "none"), g, None if r is None else r[:, a:z], None if d is None else d[:, a:z].contiguous())

    whole = run(0, M)
    for a, z in ((0, 1), (1, 3), (2, 6), (0, 8), (7, 24), (100, 164), (50, 400), (300, 1011)):
        assert same(run(a, z), whole[:, a:z]), (a, z)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 8.0])
@pytest.mark.parametrize("n,m,H", [(300, 0, 2), (1300, 0, 1), (200, 90, 2), (700, 700, 24)], ids=str)
def test_what_padding_holds_changes_no_bit(D, cap, n, m, H):
    """Tokens of no document between the others and behind them, in tiles that others share"""
    N = n + m
    d = documents(N, (N // 2, N // 3), seed=5 if H == 2 else None)
    q, k, v = normal((3, 1, H, N, D), 6)
    dt = torch.from_numpy(d).cuda()

    def run():
        o = torch.full((1, H, N, D), 7.0, dtype=torch.bfloat16, device="cuda")
        ra.rapid_attn_packed([tuple(t[:, :, a:z] for t in (q, k, v, o)) for a, z in ((0, n), (n, N)) if z > a], dt, cap=cap)
        return o

    for t in (q, k, v):
        t[:, :, d < 0] = 0
    want = run()
    for value in (NAN, float("inf"), -1.5e38):
        for t in (q, k, v):
            t[:, :, d < 0] = value
        assert same(run(), want), value
