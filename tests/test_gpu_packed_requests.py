"""What a request comes to up to its attention does not depend on what it is packed with, bit for bit: the conditioning's vectors too,
whose product is one in bf16."""
import numpy as np
import pytest
import torch

import paper_2509_22323_amd as ra
from layer_common import normal
from test_gpu_joint_layer import make as make_joint

pytestmark = pytest.mark.gpu


def same(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


@pytest.mark.parametrize("K,N", [(192, 1152), (1728, 10368), (2432, 129)], ids=str)
def test_up_to_four_rows_of_a_product_are_each_by_itself(K, N):
    x, w, b = normal((7, K), 1), normal((N, K), 2, K ** -0.5), normal((N,), 3, 0.1)
    one = torch.cat([ra.rapid_linear(x[i:i + 1], w, torch.empty((1, N), dtype=x.dtype, device="cuda"), b) for i in range(7)])
    for first, rows in ((0, 2), (1, 2), (0, 3), (4, 3), (0, 4), (3, 4), (2, 4)):
        assert same(ra.rapid_linear(x[first:first + rows], w, torch.empty((rows, N), dtype=x.dtype, device="cuda"), b), one[first:first + rows]), (first, rows)
        two = ra.rapid_linear(x[first:first + rows, None], w, torch.empty((rows, 1, N), dtype=x.dtype, device="cuda"), b)
        assert same(two[:, 0], one[first:first + rows]), (first, rows)


@pytest.mark.parametrize("H,D", [(3, 64), (27, 64)], ids=str)
def test_requests_up_to_their_attention(H, D):
    """1, 2, 4, 5, 8, 9 and 12 requests, at widths where the conditioning's product would be taken in other kernels for five rows or for nine"""
    image, text, most = 3, 2, 12
    joint = make_joint(H=H, D=D, F=16, rotate=False)[0]
    axes = [ra.RopeAxis(D // 2)]
    cond, hidden = normal((most, H * D), 5), [normal((most, n, H * D), 6 + i, 2.0) for i, n in enumerate((image, text))]

    def run(first, count):
        layer = ra.PackedLayer(joint.weights, H, D, count * image, count * text, count, axes)
        rows = [torch.arange(count, device="cuda", dtype=torch.int32).repeat_interleave(n) for n in (image, text)]
        at = [torch.arange(n, device="cuda", dtype=torch.int32).repeat(count) for n in (image, text)]
        layer.run(*(h[first:first + count].reshape(-1, H * D).clone() for h in hidden), cond[first:first + count], torch.cat(rows), torch.cat(at)[:, None])
        return [t[:count] for t in layer.mod] + [t.view(count, -1, 3, H, D) for t in layer.qkv]

    whole = run(0, most)
    assert all(torch.isfinite(t.float()).all() for t in whole)
    for first, count in ((0, 1), (7, 1), (11, 1), (3, 2), (1, 4), (0, 5), (4, 5), (2, 8), (0, 9), (3, 9)):
        for got, want in zip(run(first, count), whole):
            assert same(got, want[first:first + count]), (first, count)


def test_nine_requests_in_a_graph():
    """Three calls a stream for their conditioning; replays between eager runs, on other conditioning each time"""
    count, H, D = 9, 3, 64
    joint = make_joint(H=H, D=D, F=16, rotate=False)[0]
    layer = ra.PackedLayer(joint.weights, H, D, 3 * count, 2 * count, count)
    start = [normal((n * count, H * D), 6 + n, 2.0) for n in (3, 2)]
    hidden, cond = [t.clone() for t in start], normal((count, H * D), 5)
    document = torch.cat([torch.arange(count, device="cuda", dtype=torch.int32).repeat_interleave(n) for n in (3, 2)])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer.run(*hidden, cond, document)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run(*hidden, cond, document)
    for turn in range(3):
        cond.copy_(normal((count, H * D), 20 + turn))
        for t, s in zip(hidden, start):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in hidden]
        for t, s in zip(hidden, start):
            t.copy_(s)
        layer.run(*hidden, cond, document)
        assert all(same(a, b) for a, b in zip(got, hidden)) and not same(hidden[0], start[0])
