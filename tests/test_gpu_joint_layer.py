"""The operators together: a joint layer, dense and under a selected mask, its calls each against the oracle on what they were
given, the whole of it against fp64 throughout, captured into a graph, and inside the step-level driver."""
import numpy as np
import pytest
import torch

import paper_2509_22323_amd as ra
from layer_common import BF16_STEP, assert_within, normal, widen
from oracle import cache_oracle as co
from oracle import layer_oracle as lo
from paper_2509_22323_amd import layer as layer_module
from paper_2509_22323_amd.sampler import run_action_trace
from test_gpu_layer import modulate_bound, row_bound
from test_gpu_linear import bound as linear_bound

pytestmark = pytest.mark.gpu


def make(B=2, H=3, D=64, image=256, text=77, F=520, rotate=True, seed=1):
    C = H * D

    def stream(s):
        w = dict(mod_w=normal((6 * C, C), s, 0.5 * C ** -0.5), mod_b=normal((6 * C,), s + 1, 0.1),
                 qkv_w=normal((3 * C, C), s + 2, C ** -0.5), qkv_b=normal((3 * C,), s + 3, 0.1),
                 q_norm=normal((D,), s + 4, 0.2, 1.0), k_norm=normal((D,), s + 5, 0.2, 1.0),
                 out_w=normal((C, C), s + 6, C ** -0.5), out_b=None, ff_in_w=normal((F, C), s + 7, C ** -0.5),
                 ff_in_b=normal((F,), s + 8, 0.1), ff_out_w=normal((C, F), s + 9, F ** -0.5), ff_out_b=normal((C,), s + 10, 0.1))
        assert set(w) == set(layer_module.WEIGHTS)
        return w

    weights = stream(100 * seed), stream(100 * seed + 50)
    positions = axes = None
    if rotate:
        t = np.arange(image + text)
        p = np.stack([0 * t, np.where(t < image, t // 16, 0), np.where(t < image, t % 16, 0)], -1).astype(np.int32)
        positions, axes = torch.from_numpy(p).cuda(), [ra.RopeAxis(D // 4), ra.RopeAxis(3 * D // 8), ra.RopeAxis(3 * D // 8)]
    layer = ra.JointLayer(weights, B, H, D, image, text, positions, axes)
    hidden = normal((B, image + text, C), 7 * seed)
    return layer, hidden, normal((B, C), 8 * seed)


def halves(layer, hidden):
    image = layer.tokens[0]
    return hidden[:, :image], hidden[:, image:]


def reference(layer, hidden, cond):
    """fp64 throughout, dense attention"""
    image = layer.tokens[0]
    xs = [widen(t) for t in halves(layer, hidden)]
    table = None if layer.table is None else widen(layer.table)
    ws = [{k: None if v is None else widen(v) for k, v in w.items()} for w in layer.weights]
    mods, rows, first = [], [], 0
    for x, w in zip(xs, ws):
        B, n, C = x.shape
        m = lo.linear(widen(cond)[:, None], w["mod_w"], w["mod_b"])[:, 0].reshape(B, 6, C)
        h = lo.norm_modulate(x, m[:, 1], m[:, 0])
        q, k, v = lo.linear(h, w["qkv_w"], w["qkv_b"]).reshape(B, n, 3, layer.H, layer.D).transpose(2, 0, 3, 1, 4)
        q, k = lo.head_norm(q, w["q_norm"]), lo.head_norm(k, w["k_norm"])
        if table is not None:
            q, k = (lo.rotate(t, table[first:first + n], layer.layout) for t in (q, k))
        mods.append(m)
        rows.append((q, k, v))
        first += n
    q, k, v = (np.concatenate(t, 2) for t in zip(*rows))
    s = np.matmul(q, k.transpose(0, 1, 3, 2)) / np.sqrt(layer.D)
    p = np.exp(s - s.max(-1, keepdims=True))
    o = np.matmul(p / p.sum(-1, keepdims=True), v).transpose(0, 2, 1, 3).reshape(hidden.shape)
    out = []
    for x, m, w, a in zip(xs, mods, ws, (o[:, :image], o[:, image:])):
        x = lo.linear(a, w["out_w"], w["out_b"], "none", m[:, 2], x)
        f = lo.linear(lo.norm_modulate(x, m[:, 4], m[:, 3]), w["ff_in_w"], w["ff_in_b"], "gelu_tanh")
        out.append(lo.linear(f, w["ff_out_w"], w["ff_out_b"], "none", m[:, 5], x))
    return np.concatenate(out, 1)


@pytest.mark.parametrize("kw", [dict(), dict(rotate=False, text=1), dict(D=128, H=2, B=1, image=128, text=200, F=304)], ids=str)
def test_every_call_of_a_layer(kw, monkeypatch):
    layer, hidden, cond = make(**kw)
    count = [0]

    def num(t):
        return None if t is None else widen(t)

    def linear(x, weight, out, bias=None, activation="none", gate=None, residual=None, workspace=None):
        args = [num(t.view(t.shape[0], -1, t.shape[-1])) for t in (x, residual if residual is not None else out)]
        three = [args[0], num(weight), num(bias), activation, num(gate), args[1] if residual is not None else None]
        if x.dim() == 2:
            three[0] = num(x)[None]
        real_linear(x, weight, out, bias, activation, gate, residual, workspace)
        want = lo.linear(*three)
        assert_within(out.view(want.shape), want, linear_bound(*three, want), "linear")
        count[0] += 1

    def modulate(x, out, scale=None, shift=None, eps=1e-6):
        real_modulate(x, out, scale, shift, eps)
        want = lo.norm_modulate(num(x), num(scale), num(shift), eps)
        assert_within(out, want, modulate_bound(num(x), num(scale), want), "norm")
        count[0] += 1

    def qk(segments, weights, table, layout, eps):
        before = [[num(t) for t in seg[:2]] for seg in segments]
        real_qk(segments, weights, table, layout, eps)
        first = 0
        for seg, two, w in zip(segments, before, weights):
            for t, u, g in zip(seg[2:], two, w):
                v = lo.head_norm(u, num(g), eps)
                if table is not None:
                    v = lo.rotate(v, num(table)[first:first + u.shape[2]], layout)
                assert_within(t, v, row_bound(u, num(g), v, True, table is not None), "queries and keys")
            first += u.shape[2]
        count[0] += 1

    real_linear, real_modulate, real_qk = ra.rapid_linear, ra.rapid_norm_modulate, ra.rapid_qk_norm_rope
    want = reference(layer, hidden, cond)
    monkeypatch.setattr(layer_module._b, "rapid_linear", linear)
    monkeypatch.setattr(layer_module._b, "rapid_norm_modulate", modulate)
    monkeypatch.setattr(layer_module._b, "rapid_qk_norm_rope", qk)
    layer.run(*halves(layer, hidden), cond)
    assert count[0] == 2 * 7 + 1
    # Along the longest way a value is rounded to bf16 eleven times (conditioning, norm, projection, queries, scores' weights,
    # attention, hidden state, norm, feed-forward's middle, hidden state, and once more where a gate is), each by half a step
    # at most, in the mean square by less than half of that; operators neither grow nor shrink the relative error much.
    d = widen(hidden) - want
    assert np.sqrt((d * d).sum() / (want * want).sum()) <= 12 * BF16_STEP / 2


@pytest.mark.parametrize("a_sparse", [0, 2])
def test_a_captured_layer(a_sparse):
    layer, hidden, cond = make(image=384, seed=3)
    start = hidden.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.run(*halves(layer, hidden), cond, a_sparse)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run(*halves(layer, hidden), cond, a_sparse)
    for turn in range(3):
        start.add_(0.25 * turn)
        hidden.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        got = hidden.clone()
        hidden.copy_(start)
        layer.run(*halves(layer, hidden), cond, a_sparse)
        torch.cuda.synchronize()
        assert torch.isfinite(got).all() and torch.equal(got, hidden)


def test_lengths_of_prompts():
    """Text behind a sample's length changes nothing of its image tokens."""
    layer, hidden, cond = make(text=100, seed=4)
    lens = torch.tensor([256 + 100, 256 + 40], dtype=torch.int32, device="cuda")
    other = hidden.clone()
    other[1, 256 + 40:] = normal(other[1, 256 + 40:].shape, 5, 30.0)
    for x in (hidden, other):
        layer.run(*halves(layer, x), cond, 0, lens)
    assert torch.equal(hidden[:, :256 + 40], other[:, :256 + 40])


def test_driver_runs_layers():
    layer, hidden, cond = make(seed=6)
    B = layer.B
    x = hidden.reshape(B, -1).clone()
    delta, out = torch.zeros_like(x), torch.zeros_like(x)
    trace = [(0, 0), (1, 0), (0, 1), (1, 0)]
    res = run_action_trace(trace, None, None, None, None, 2, 128, None, None, x, delta, out, layer=layer, conditioning=cond)
    assert [s["kind"] for s in res.steps] == ["full", "cached", "sparse-1", "cached"]
    assert res.calls == {"JointLayer.run": 4, "rapid_cache_reuse": 2, "rapid_cache_store": 2}
    want = hidden.clone()
    for _ in range(2):
        layer.run(*halves(layer, want), cond, 1)
    bits = lambda t: t.reshape(B, -1).view(torch.int16).cpu().numpy().view(np.uint16)
    step = co.cache_store(bits(want), bits(x))
    np.testing.assert_array_equal(bits(delta), step)
    np.testing.assert_array_equal(bits(out), co.cache_reuse(bits(x), step))
    with pytest.raises(ValueError):
        run_action_trace([(1, 0)], None, None, None, None, 1, 128, None, None, x, delta, out, layer=layer, conditioning=cond)


def test_two_layers_at_once():
    """Layers with buffers of their own on two streams, their calls interleaved: the bits of one after the other."""
    pairs = [make(seed=s) for s in (11, 12)]
    starts = [h.clone() for _, h, _ in pairs]
    for layer, hidden, cond in pairs:
        layer.run(*halves(layer, hidden), cond, 1)
    want = [h.clone() for _, h, _ in pairs]
    streams = [torch.cuda.Stream() for _ in pairs]
    for _ in range(3):
        for (_, hidden, _), start in zip(pairs, starts):
            hidden.copy_(start)
        torch.cuda.synchronize()
        for stream, (layer, hidden, cond) in zip(streams, pairs):
            with torch.cuda.stream(stream):
                layer.run(*halves(layer, hidden), cond, 1)
        torch.cuda.synchronize()
        for (_, hidden, _), w in zip(pairs, want):
            assert torch.equal(hidden, w)


def test_products_on_two_streams_take_workspaces_of_their_own():
    x, w = normal((2, 150, 4096), 1), normal((320, 4096), 2, 1 / 64)
    assert ra.rapid_linear_workspace_bytes(300, 320, 4096) > 0
    want = ra.rapid_linear(x, w, torch.empty((2, 150, 320), dtype=x.dtype, device="cuda"))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for i in range(8):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(ra.rapid_linear(x, w, torch.empty_like(want)))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_padding_that_is_not_a_number():
    """Text rows behind a sample's length that hold no numbers: nothing of them reaches the rows before."""
    layer, hidden, cond = make(text=100, seed=5)
    lens = torch.tensor([256 + 100, 256 + 40], dtype=torch.int32, device="cuda")
    other = hidden.clone()
    other[1, 256 + 40:] = float("nan")
    for x in (hidden, other):
        layer.run(*halves(layer, x), cond, 0, lens)
    assert torch.isfinite(hidden).all()
    assert torch.equal(hidden[:, :256 + 40], other[:, :256 + 40]) and torch.equal(hidden[0], other[0])
