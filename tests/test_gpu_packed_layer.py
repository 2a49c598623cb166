"""The operators of packed sequences together: a layer in 8 bits over packed requests, its calls each against the oracle on what they
were given, requests packed and alone, padding, graphs, other streams and two layers at once."""
import numpy as np
import pytest
import torch

import paper_2509_22323_amd as ra
from layer_common import BF16_STEP, assert_within, normal, widen
from oracle import layer_oracle as lo
from oracle import packed_oracle as po
from paper_2509_22323_amd import layer as layer_module
from test_gpu_attn_packed import bound as attention_bound
from test_gpu_int8 import assert_normed, bound as linear_bound
from test_gpu_joint_layer import make as make_joint

pytestmark = pytest.mark.gpu

REQUESTS = ((100, 20), (64, 31), (1, 7), (60, 1))      # image and text tokens of each


def make(H=3, D=64, F=528, requests=REQUESTS, pads=(5, 9), rotate=True, seed=1, documents=None):
    """(layer, hidden states of both streams, arguments of a run)"""
    weights = make_joint(H=H, D=D, F=F, seed=seed)[0].weights
    lengths = [sum(r[i] for r in requests) + pads[i] for i in range(2)]
    axes = [ra.RopeAxis(D // 4), ra.RopeAxis(3 * D // 8), ra.RopeAxis(3 * D // 8)] if rotate else None
    layer = ra.PackedLayer(weights, H, D, *lengths, documents or len(requests), axes)
    C = H * D
    hidden = [normal((n, C), 7 * seed + i, 2.0) for i, n in enumerate(lengths)]
    d = [np.concatenate([np.full(r[i], j) for j, r in enumerate(requests)] + [np.full(pads[i], -1)]) for i in range(2)]
    at = [np.concatenate([np.arange(r[i]) for r in requests] + [np.zeros(pads[i], int)]) for i in range(2)]
    p = np.concatenate([np.stack([0 * at[0], at[0] // 8, at[0] % 8], -1), np.zeros((lengths[1], 3), int)])
    args = dict(conditioning=normal((len(requests), C), 8 * seed), document=torch.from_numpy(np.concatenate(d).astype(np.int32)).cuda())
    if rotate:
        args["positions"] = torch.from_numpy(p.astype(np.int32)).cuda()
    return layer, hidden, args


@pytest.mark.parametrize("kw,run", [(dict(), dict()), (dict(rotate=False, pads=(0, 0)), dict(cap=5.0)), (dict(H=2, D=128, F=304), dict(text_first=True)),
                                    (dict(requests=((300, 40),), pads=(1, 0)), dict())], ids=str)
def test_every_call_of_a_layer(kw, run, monkeypatch):
    layer, hidden, args = make(**kw)
    if run.pop("text_first", False):
        args["order"] = (torch.arange(sum(layer.tokens), device="cuda") < layer.tokens[0]).int()
    calls = []

    def num(t):
        return None if t is None else widen(t)

    def quantize(x, q, scale):
        real["rapid_quantize_rows"](x, q, scale)
        want = po.quantize(num(x))
        assert np.array_equal(num(q), want[0]) and np.array_equal(scale.cpu().numpy(), want[1].astype(np.float32))
        calls.append("quantize")
        return q, scale

    def norm(x, q, q_scale, scale, shift, eps, document):
        real["rapid_norm_modulate_int8"](x, q, q_scale, scale, shift, eps, document)
        d = document.cpu().numpy()[None]
        assert_normed(po.norm_modulate(num(x)[None], num(scale), num(shift), eps, d), (q[None], q_scale[None]), d >= 0)
        calls.append("norm")

    def linear(x, x_scale, weight, w_scale, out, bias=None, activation="none", gate=None, residual=None, document=None, workspace=None):
        before = num(out)
        four = [num(t) for t in (x[None], x_scale[None], weight, w_scale)]
        b, g, r = num(bias), num(gate), None if residual is None else num(residual)[None]
        d = None if document is None else document.cpu().numpy()[None]
        real["rapid_linear_int8"](x, x_scale, weight, w_scale, out, bias, activation, gate, residual, document, workspace)
        want = po.linear(*four, b, activation, g, r, d)
        e = linear_bound(po.linear(*four), b, activation, None if g is None else g[d.clip(0)], r, want)
        rows = np.ones(out.shape[0], bool) if d is None else d[0] >= 0
        assert_within(out[torch.from_numpy(rows).cuda()], want[0][rows], e[0][rows], "linear")
        assert np.array_equal(num(out)[~rows], before[~rows])
        calls.append("linear")

    def attend(segments, document, order, cap, workspace):
        real["rapid_attn_packed"](segments, document, order, cap, workspace=workspace)
        q, k, v, got = (np.concatenate([num(s[i]) for s in segments], 2) for i in range(4))
        d, o = document.cpu().numpy()[None], None if order is None else order.cpu().numpy()[None]
        want, p = po.attention(q, k, v, d, o, cap)
        e = attention_bound(q, k, v, p, want, cap, layer.D ** -0.5, po.visible(d, o))
        assert (np.abs(got - want) <= e).all()
        calls.append("attention")

    real = {n: getattr(layer_module._b, n) for n in ("rapid_quantize_rows", "rapid_norm_modulate_int8", "rapid_linear_int8", "rapid_attn_packed")}
    for n, f in zip(real, (quantize, norm, linear, attend)):
        monkeypatch.setattr(layer_module._b, n, f)
    start = [t.clone() for t in hidden]
    assert layer.run(*hidden, **args, **run)[0] is hidden[0]
    assert calls == ["norm", "linear"] * 2 + ["attention"] + ["quantize", "linear", "norm", "linear", "quantize", "linear"] * 2
    for t, s, d in zip(hidden, start, args["document"].split(list(layer.tokens))):
        assert torch.equal(t[d < 0], s[d < 0]) and not torch.equal(t[d >= 0], s[d >= 0]) and torch.isfinite(t).all()


def test_a_layer_is_near_the_one_in_bf16():
    """One request, the same weights in bf16: 8 bits a row and a column are 127 steps up to the largest element.  A product of K terms of
    rows and columns with independent roundings of up to half a step (largest / 254) is off by about sqrt(K) / sqrt(12) (step_x |w| + step_w |x|),
    1.4 % of its size at 4 standard deviations a largest element; four products behind each other on the residual stream: 8 % covers
    them, and the attention between them, twice over."""
    joint, hidden, cond = make_joint(B=1, H=3, D=64, image=256, text=77, F=528, rotate=False, seed=3)
    packed = ra.PackedLayer(joint.weights, 3, 64, 256, 77, 1)
    a, b = [hidden[0, :256].clone(), hidden[0, 256:].clone()], [hidden[:, :256].clone(), hidden[:, 256:].clone()]
    packed.run(*a, cond, torch.zeros(333, dtype=torch.int32, device="cuda"))
    joint.run(*b, cond)
    for x, y, h in zip(a, b, (hidden[0, :256], hidden[0, 256:])):
        moved = (y[0].double() - h.double()).norm()
        assert (x.double() - y[0].double()).norm() <= 0.08 * moved


def test_requests_packed_and_alone():
    """What a request comes to is the same but for the order of the sums of its attention: weights in other tiles are rounded to bf16
    against other references, which the quantisation of the next rows can carry over a border."""
    layer, hidden, args = make(pads=(0, 0))
    start = [t.clone() for t in hidden]
    layer.run(*hidden, **args)
    at = [0, 0]
    joint = make_joint(H=3, D=64, F=528, seed=1)[0]
    for j, (n, m) in enumerate(REQUESTS):
        rows = [slice(a, a + k) for a, k in zip(at, (n, m))]
        one = ra.PackedLayer(joint.weights, 3, 64, n, m, 1, layer.axes)
        own = [s[r].clone() for s, r in zip(start, rows)]
        p = torch.cat([args["positions"][:layer.tokens[0]][rows[0]], args["positions"][layer.tokens[0]:][rows[1]]])
        one.run(*own, args["conditioning"][j:j + 1], torch.zeros(n + m, dtype=torch.int32, device="cuda"), p)
        for got, want, r, s in zip(hidden, own, rows, start):
            moved = (want.double() - s[r].double()).norm()
            assert (got[r].double() - want.double()).norm() <= 0.01 * moved
        at = [a + k for a, k in zip(at, (n, m))]


def test_a_captured_layer():
    """Replays between eager runs, on new hidden states, conditioning and packing (the same buffers) each time"""
    layer, hidden, args = make()
    start = [t.clone() for t in hidden]
    layer.run(*hidden, **args)
    eager = [t.clone() for t in hidden]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer.run(*hidden, **args)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run(*hidden, **args)
    for turn in range(3):
        for t, s in zip(hidden, start):
            t.copy_(s * (1 + turn))
        if turn == 2:
            args["document"].copy_(args["document"].flip(0))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in hidden]
        for t, s in zip(hidden, start):
            t.copy_(s * (1 + turn))
        layer.run(*hidden, **args)
        assert all(torch.equal(a, b) for a, b in zip(got, hidden))
        if turn == 0:
            assert all(torch.equal(a, b) for a, b in zip(got, eager))


def test_two_layers_on_two_streams():
    layers = [make(seed=s) for s in (1, 2)]
    want = []
    for layer, hidden, args in layers:
        h = [t.clone() for t in hidden]
        layer.run(*h, **args)
        want.append(h)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for (layer, hidden, args), s in zip(layers, streams):
        with torch.cuda.stream(s):
            layer.run(*hidden, **args)
    torch.cuda.synchronize()
    for (_, hidden, _), w in zip(layers, want):
        assert all(torch.equal(a, b) for a, b in zip(hidden, w))


def test_fewer_requests_than_the_layer_was_made_for():
    layer, hidden, args = make(documents=9)
    other, second, _ = make()
    layer.run(*hidden, **args)
    other.run(*second, **args)
    assert all(torch.equal(a, b) for a, b in zip(hidden, second))
