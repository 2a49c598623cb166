"""The norm under the conditioning, the norm and rotation of queries and keys and the table of angles against the fp64 oracle."""
import numpy as np
import pytest
import torch

import paper_2509_22323_amd as ra
from layer_common import BF16_STEP, NAN, assert_within, inside, normal, untouched_around, widen
from oracle import layer_oracle as lo

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------- norm under scale and shift
def modulate_bound(x, scale, want):
    """A sum of C terms in fp32, lane by lane and then over lanes, is off by at most (C / 64 + 16) roundings of the terms'
    absolute sum: the mean by d = that / C.  Each deviation carries d and one rounding of its own and of x; the mean square
    deviation, its root and quotient 2 (d / sigma) + (C / 64 + 20) 2^-24 relative.  Then scale and shift: three roundings."""
    C = x.shape[-1]
    steps = (C / 64 + 16) * 2.0 ** -24
    sigma = np.sqrt(x.var(-1, keepdims=True) + 1e-6)
    d = steps * np.abs(x).mean(-1, keepdims=True) + 2.0 ** -24 * np.abs(x)
    z = np.abs(x - x.mean(-1, keepdims=True)) / sigma
    factor = 1.0 if scale is None else np.abs(1.0 + scale[:, None])
    d_row = d.max(-1, keepdims=True)
    e = factor * (d / sigma + z * (2.0 * d_row / sigma + steps + 6 * 2.0 ** -24)) + 2.0 ** -23 * np.abs(want)
    return e + BF16_STEP * (np.abs(want) + e) + 2.0 ** -134


MODULATE = [(1, 1, 8), (1, 5, 64), (2, 3, 72), (1, 7, 512), (3, 9, 520), (1, 33, 1024), (2, 333, 1536), (1, 4, 2048), (1, 77, 2432),
            (2, 10, 4096), (1, 6, 4104), (1, 3, 8192), (2, 5, 8200), (1, 2, 16384), (300, 1, 128), (40, 7, 1536)]


@pytest.mark.parametrize("affine", [False, True])
@pytest.mark.parametrize("size", MODULATE, ids=str)
def test_norm_modulate(size, affine):
    B, n, C = size
    xt = normal(size, 1, 3.0, 5.0)
    x, _ = inside(xt, 1, 2, 8)
    v = normal((B, 6, C), 2, 0.5)
    scale, shift = (v[:, 3], v[:, 4]) if affine else (None, None)
    out, big = inside(torch.full(size, NAN, dtype=torch.bfloat16, device="cuda"), 2, 1, 16)
    assert ra.rapid_norm_modulate(x, out, scale, shift) is out
    s, t = (widen(scale), widen(shift)) if affine else (None, None)
    want = lo.norm_modulate(widen(xt), s, t)
    assert_within(out, want, modulate_bound(widen(xt), s, want))
    assert untouched_around(out, big)
    first = out.clone()
    ra.rapid_norm_modulate(x, x, scale, shift)                                     # in place
    assert torch.equal(x, first)


def test_norm_modulate_one_vector_for_all_and_constant_rows():
    x = normal((4, 6, 256), 3)
    x[1, 2] = 3.0                                                                  # no deviation: the shift alone
    v = normal((2, 256), 4)
    out = ra.rapid_norm_modulate(x, torch.empty_like(x), v[0], v[1])
    s, t = (np.broadcast_to(widen(a), (4, 256)) for a in v)
    want = lo.norm_modulate(widen(x), s, t)
    assert_within(out, want, modulate_bound(widen(x), s, want))
    assert torch.equal(out[1, 2], v[1])
    flat = ra.rapid_norm_modulate(x.view(24, 256), torch.empty_like(x).view(24, 256), v[0], v[1])
    assert torch.equal(flat.view(4, 6, 256), out)
    x[0, 0, 5] = NAN                                                               # stays in its row
    again = ra.rapid_norm_modulate(x, torch.empty_like(x), v[0], v[1])
    assert torch.isnan(again[0, 0]).all() and torch.equal(again.view(24, 256)[1:], flat[1:])


def test_norm_modulate_far_mean():
    """A mean of 1000 deviations: in one pass over squares no digit would be left."""
    x = normal((1, 5, 1536), 6, 1.0, 0.0)
    x = (x.float() + 1024.0).to(torch.bfloat16)                                    # steps of 8 around 1024
    x[..., ::2] += 16
    out = ra.rapid_norm_modulate(x, torch.empty_like(x))
    want = lo.norm_modulate(widen(x))
    assert_within(out, want, modulate_bound(widen(x), None, want))


# ------------------------------------------------------------------------------------- queries and keys
def tensors(layout, B, H, n, D, seed, scale=2.0):
    """(q, k) of a segment: head-major, token-major or slices of a fused projection"""
    if layout == "head":
        t = normal((2, B, H, n, D), seed, scale)
        return t[0], t[1]
    if layout == "token":
        t = normal((2, B, n, H, D), seed, scale).transpose(2, 3)
        return t[0], t[1]
    t = normal((B, n, 3, H, D), seed, scale).permute(2, 0, 3, 1, 4)
    return t[0], t[1]


def angles(N, rot, seed, B=None):
    rng = np.random.default_rng(seed)
    a = rng.uniform(-4.0, 4.0, (N, rot // 2) if B is None else (B, N, rot // 2))
    return torch.from_numpy(np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)).cuda()


def row_bound(u, weight, want, norm, rot):
    """Sum of D squares: (D / 8 + 4) roundings at most, half of that relative error through the root, quotient and root and
    weight four more; a pair's turn: two products and a sum, of at most the pair's absolute sum, which any element of the row
    times two bounds together with the other one of the pair."""
    steps = (u.shape[-1] / 8 + 12) * 2.0 ** -24 if norm else 0.0
    v = np.abs(lo.head_norm(u, weight)) if norm else np.abs(u)
    e = v.max(-1, keepdims=True) * 2.0 * (steps + 3 * 2.0 ** -24) if rot else v * steps
    return e + BF16_STEP * (np.abs(want) + e) + 2.0 ** -134


QK = [  # B, H, n0, n1 (0: one segment), D, rot, layout of the pairs, of the tensors
    (1, 1, 1, 0, 64, 64, "interleaved", "head"), (1, 2, 1, 1, 128, 128, "half", "fused"), (1, 24, 1, 0, 128, 128, "interleaved", "fused"),
    (2, 3, 17, 5, 64, 32, "half", "head"), (2, 5, 33, 0, 128, 64, "interleaved", "token"), (3, 4, 7, 9, 64, 16, "interleaved", "fused"),
    (1, 38, 12, 3, 64, 64, "half", "fused"), (2, 24, 64, 77, 128, 128, "interleaved", "fused"), (1, 7, 130, 1, 128, 48, "half", "token"),
    (1, 6, 50, 0, 128, 112, "half", "head"), (4, 1, 9, 0, 64, 48, "interleaved", "token"), (1, 9, 256, 31, 128, 16, "half", "fused"),
    (2, 24, 333, 0, 64, 0, "interleaved", "fused"), (1, 3, 5, 6, 128, 0, "half", "head"),
]


@pytest.mark.parametrize("case", QK, ids=str)
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("per_sample", [False, True])
def test_qk_rows(case, norm, per_sample):
    B, H, n0, n1, D, rot, pairs, layout = case
    if not norm and rot == 0:
        pytest.skip("nothing to do")
    lengths = [n for n in (n0, n1) if n]
    table = angles(sum(lengths), rot, 9, B if per_sample else None) if rot else None
    segments, weights, wants = [], [], []
    first = 0
    for i, n in enumerate(lengths):
        q, k = tensors(layout, B, H, n, D, 10 + i)
        outs = tensors("token", B, H, n, D, 0, NAN) if layout == "fused" else tensors(layout, B, H, n, D, 0, NAN)
        segments.append((q, k, *outs))
        weights.append((normal((D,), 20 + i, 0.2, 1.0), None if i else normal((D,), 30, 0.2, 1.0)))
        for t, w in zip((q, k), weights[i]):
            u, w = widen(t), None if w is None else widen(w)
            v = lo.head_norm(u, w) if norm else u
            if rot:
                tab = widen(table)[..., first:first + n, :, :]
                v = lo.rotate(v, tab, pairs)
            wants.append((v, row_bound(u, w, v, norm, rot)))
        first += n

    def call(segs):
        return ra.rapid_qk_norm_rope(segs, weights, table, pairs) if norm else ra.rapid_rope(segs, table, pairs)

    for got, (want, e) in zip(call(segments), wants):
        assert_within(got, want, e)
    kept = [t.clone() for seg in segments for t in seg[2:]]
    call([(q, k, q, k) for q, k, _, _ in segments])                                # in place
    for seg, a, b in zip(segments, kept[::2], kept[1::2]):
        assert torch.equal(seg[0], a) and torch.equal(seg[1], b)


def test_values_behind_fused_queries_and_keys_are_left_alone():
    B, n, H, D = 2, 19, 5, 64
    t = normal((B, n, 3, H, D), 41)
    v = t[:, :, 2].clone()
    q, k = (t.permute(2, 0, 3, 1, 4)[i] for i in (0, 1))
    ra.rapid_qk_norm_rope([(q, k, q, k)], None, angles(n, 64, 2))
    assert torch.equal(t[:, :, 2], v)


def test_unturned_elements_and_special_values():
    """Elements behind the rotated part keep their bits in the rotation alone, infinities and NaN stay in their pair."""
    B, H, n, D, rot = 1, 2, 9, 128, 32
    for pairs in ("interleaved", "half"):
        q, k = tensors("head", B, H, n, D, 50)
        q[0, 0, 3, 100], q[0, 1, 4, 2], k[0, 0, 0, 127] = NAN, NAN, float("inf")
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        ra.rapid_rope([(q, k, qo, ko)], angles(n, rot, 3), pairs)
        assert torch.equal(qo[..., rot:].view(torch.int16), q[..., rot:].view(torch.int16)) and torch.equal(ko[..., rot:], k[..., rot:])
        lost = torch.isnan(qo[0, 1, 4])
        assert lost.sum() == 2 and lost[2] and lost[3 if pairs == "interleaved" else 2 + rot // 2]


def test_zero_rows_stay_zero_under_eps():
    q, k = tensors("head", 1, 2, 8, 64, 60)
    q[0, 1, 5] = 0
    qo, ko = ra.rapid_qk_norm_rope([(q, k, torch.empty_like(q), torch.empty_like(k))], None, angles(8, 64, 1))
    assert (qo[0, 1, 5] == 0).all() and torch.isfinite(ko).all()


# ------------------------------------------------------------------------------------- table
AXES = [
    [dict(dim=64, theta=10000.0)], [dict(dim=16, theta=10000.0), dict(dim=56, theta=10000.0), dict(dim=56, theta=10000.0)],
    [dict(dim=32, theta=100.0, scaling="linear", factor=2.5), dict(dim=32, theta=10000.0, scaling="ntk", factor=4.0)],
    [dict(dim=128, theta=500000.0, scaling="by_parts", factor=8.0, original_length=4096.0, beta_fast=32.0, beta_slow=1.0)],
    [dict(dim=2, theta=10000.0)] * 8, [dict(dim=4, theta=10000.0, scaling="ntk", factor=3.0), dict(dim=12, theta=7.0)],
]


@pytest.mark.parametrize("axes", AXES, ids=lambda a: "-".join(str(x["dim"]) + x.get("scaling", "") for x in a))
@pytest.mark.parametrize("shape", [(1,), (7,), (4609,), (3, 50)], ids=str)
@pytest.mark.parametrize("magnitude", [1.0, 1.2])
def test_table(axes, shape, magnitude):
    rng = np.random.default_rng(7)
    p = rng.integers(-5000, 70000, (*shape, len(axes))).astype(np.int32)
    p.reshape(-1)[0] = 1 << 24
    p.reshape(-1)[-1] = 0 if p.size > 1 else p.reshape(-1)[-1]
    pairs = sum(a["dim"] for a in axes) // 2
    table = torch.full((*shape, pairs, 2), NAN, device="cuda")
    assert ra.rapid_rope_table(torch.from_numpy(p).cuda(), [ra.RopeAxis(**a) for a in axes], table, magnitude) is table
    want = lo.table(p, axes, magnitude)
    # half a step of fp32; the angle's frequency, product and reduction: four roundings of fp64 of up to 2^24 radians
    e = 2.0 ** -24 * np.abs(want) + magnitude * 4 * 2.0 ** -53 * 2.0 ** 24
    assert_within(table, want, e)


def test_far_positions_keep_their_angle():
    """Positions that fp32 does not hold: odd numbers beyond 2^24."""
    p = torch.tensor([[(1 << 24) + 1], [(1 << 26) - 1], [-(1 << 26) + 1]], dtype=torch.int32, device="cuda")
    axis = dict(dim=32, theta=10000.0)
    table = ra.rapid_rope_table(p, [ra.RopeAxis(**axis)], torch.empty(3, 16, 2, device="cuda"))
    want = lo.table(p.cpu().numpy(), [axis])
    assert_within(table, want, 2.0 ** -24 * np.abs(want) + 4 * 2.0 ** -53 * 2.0 ** 26)


# ------------------------------------------------------------------------------------- graphs and streams
def test_captured_calls_repeat_what_eager_calls_do():
    B, n, H, D, C = 2, 70, 4, 64, 256
    x, w = normal((B, n, C), 1), normal((3 * C, C), 2, C ** -0.5)
    wo, v = normal((C, C), 3, C ** -0.5), normal((B, 6, C), 4, 0.3)
    h, qkv, y = torch.empty_like(x), torch.empty((B, n, 3, H, D), dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    positions = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].contiguous()
    table = torch.empty(n, D // 2, 2, device="cuda")
    axes = [ra.RopeAxis(D)]
    ws = torch.empty(max(ra.rapid_linear_workspace_bytes(B * n, 3 * C, C), ra.rapid_linear_workspace_bytes(B * n, C, C), 16),
                     dtype=torch.uint8, device="cuda")
    q, k, _ = qkv.permute(2, 0, 3, 1, 4)

    def step():
        ra.rapid_rope_table(positions, axes, table)
        ra.rapid_norm_modulate(x, h, v[:, 0], v[:, 1])
        ra.rapid_linear(h, w, qkv.view(B, n, 3 * C), workspace=ws)
        ra.rapid_qk_norm_rope([(q, k, q, k)], None, table)
        ra.rapid_linear(qkv[:, :, 0].reshape(B, n, C), wo, y, None, "silu", v[:, 2], x, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                      # another stream than the tensors'
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        x.copy_(normal((B, n, C), 100 + turn))
        positions.add_(turn)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (table, h, qkv, y)]
        for t in (table, h, qkv, y):
            t.fill_(NAN)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (table, h, qkv, y)))


# ------------------------------------------------------------------------------------- large tensors, both forms of the binding
def test_offsets_beyond_32_bits():
    n, C = 1500000, 1536                                                           # 4.6 GB
    x = torch.zeros((1, n, C), dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 699050, 699051, 1398101, n - 1], device="cuda")
    x[0, rows] = normal((5, C), 71)
    x = ra.rapid_norm_modulate(x, torch.full_like(x, NAN))
    want = lo.norm_modulate(widen(normal((5, C), 71)))
    assert_within(x[0, rows], want, modulate_bound(widen(normal((5, C), 71)), None, want))
    x[0, rows] = 0
    assert not x.any()
    del x
    H, n, D = 24, 700000, 128                                                      # 4.3 GB each of q and k
    t = torch.zeros((2, 1, H, n, D), dtype=torch.bfloat16, device="cuda")
    at = [(0, 0), (7, 599186), (23, n - 1), (12, 1), (11, n - 2)]
    u = normal((5, 2, D), 72, 2.0)
    for (h, r), v in zip(at, u):
        t[:, 0, h, r] = v
    table = torch.zeros((n, 64, 2), device="cuda")
    some = angles(5, 128, 73)
    for (h, r), v in zip(at, some):
        table[r] = v
    q, k = ra.rapid_qk_norm_rope([(t[0], t[1], t[0], t[1])], None, table)
    for (h, r), v, a in zip(at, widen(u), widen(some)):
        for got, one in zip((q, k), v):
            want = lo.rotate(lo.head_norm(one)[None, None, None], a[None], "interleaved")[0, 0, 0]
            assert_within(got[0, h, r], want, row_bound(one, None, want, True, 128))


def calls():
    """Every operator as (call, its outputs), in ways that the native form takes and in ways that it leaves to Python's."""
    x, w, g, r = normal((2, 9, 64), 1), normal((40, 64), 2, 0.1), normal((2, 40), 3), normal((2, 9, 40), 4)
    b = normal((40,), 5)
    out, y = torch.empty_like(r), torch.empty_like(x)
    v = normal((2, 2, 64), 6)
    q = normal((4, 2, 3, 9, 64), 7)
    table = torch.empty(9, 32, 2, device="cuda")
    p = torch.arange(9, dtype=torch.int32, device="cuda")[:, None].contiguous()
    axes = [ra.RopeAxis(64, 100.0, "ntk", 2.0)]
    fixed = angles(9, 32, 8)
    norms = [(normal((64,), 9), None)]
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    return [
        (lambda: ra.rapid_linear(x, w, out, b, "silu", g, r), [out]), (lambda: ra.rapid_linear(x, w, out, workspace=ws), [out]),
        (lambda: ra.rapid_linear(x[0], w, out[1], None, "gelu_tanh", g[1], r[0]), [out]),
        (lambda: ra.rapid_norm_modulate(x, y, v[:, 0], v[:, 1]), [y]), (lambda: ra.rapid_norm_modulate(x[1], y[0], v[0, 0], v[0, 1], eps=0), [y]),
        (lambda: ra.rapid_rope_table(p, axes, table), [table]), (lambda: ra.rapid_rope_table(p, iter(axes), table, magnitude=2), [table]),
        (lambda: ra.rapid_rope([(q[0], q[1], q[2], q[3])], fixed, "half"), [q]),
        (lambda: ra.rapid_rope(((q[0], q[1], q[2], q[3]),), fixed[None].repeat(2, 1, 1, 1)), [q]),
        (lambda: ra.rapid_qk_norm_rope([[q[0], q[1], q[2], q[3]]], norms, fixed), [q]),
        (lambda: ra.rapid_qk_norm_rope([(q[0], q[1], q[2], q[3])]), [q]),
    ]


def test_both_forms_of_the_binding_agree(monkeypatch):
    results = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(ra.binding, "_native", ra.binding._NoNative())
        results.append([])
        for call, outs in calls():
            call()
            results[-1] += [t.clone() for t in outs]
    assert all(torch.equal(a, b) for a, b in zip(*results)) and len(results[0]) == 11


@pytest.mark.parametrize("native", [True, False])
def test_refusals_of_tensors_that_do_not_fit(native, monkeypatch):
    if not native:
        monkeypatch.setattr(ra.binding, "_native", ra.binding._NoNative())
    x, w, out = normal((2, 9, 64), 1), normal((40, 64), 2), torch.empty((2, 9, 40), dtype=torch.bfloat16, device="cuda")
    q = normal((1, 2, 9, 64), 3)
    table = angles(9, 64, 1)
    p = torch.zeros((9, 1), dtype=torch.int32, device="cuda")
    refused = [
        (TypeError, lambda: ra.rapid_linear(x.float(), w, out)), (TypeError, lambda: ra.rapid_linear(x, w.cpu(), out)),
        (TypeError, lambda: ra.rapid_linear(x, w, out, b"bias")), (TypeError, lambda: ra.rapid_linear(x[:, :, ::2], w[:, :32], out)),
        (ValueError, lambda: ra.rapid_linear(x, w[:, :56], out)), (ValueError, lambda: ra.rapid_linear(x, w, out[:1])),
        (ValueError, lambda: ra.rapid_linear(x, w, out, w[0])), (ValueError, lambda: ra.rapid_linear(x, w, out, activation="relu")),
        (ValueError, lambda: ra.rapid_linear(x, w, out, gate=out[0])), (ValueError, lambda: ra.rapid_linear(x, w, out, residual=out[:, :8])),
        (TypeError, lambda: ra.rapid_linear(x, w, out, workspace=4)), (ra.RapidAttnError, lambda: ra.rapid_linear(x[..., :60], w[:, :60], out)),
        (ra.RapidAttnError, lambda: ra.rapid_linear(x, w, out[:, :1].expand(2, 9, 40))),
        (ValueError, lambda: ra.rapid_norm_modulate(x, x, w[0])), (ValueError, lambda: ra.rapid_norm_modulate(x, x[:, :8])),
        (ra.RapidAttnError, lambda: ra.rapid_norm_modulate(x[..., 1:57], x[..., 1:57])),
        (TypeError, lambda: ra.rapid_rope_table(p.long(), [ra.RopeAxis(64)], table)), (ValueError, lambda: ra.rapid_rope_table(p, [ra.RopeAxis(32)], table)),
        (ValueError, lambda: ra.rapid_rope_table(p, [ra.RopeAxis(64)] * 2, table)), (ra.RapidAttnError, lambda: ra.rapid_rope_table(p, [ra.RopeAxis(64, -1.0)], table)),
        (ValueError, lambda: ra.rapid_rope([(q, q, q, q)], table[:8])), (ra.RapidAttnError, lambda: ra.rapid_rope([(q, q, q, q)], table)),
        (ValueError, lambda: ra.rapid_rope([(q, q[:, :1], q, q)], table)), (TypeError, lambda: ra.rapid_rope([(q, q, q, q)], table.half())),
        (ValueError, lambda: ra.rapid_qk_norm_rope([(q, q, q, q)], [])), (ValueError, lambda: ra.rapid_qk_norm_rope([(q, q, q, q)], [(w[0, :32].contiguous(), None)])),
    ]
    for kind, call in refused:
        with pytest.raises(kind):
            call()
