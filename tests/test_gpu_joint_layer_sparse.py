"""The Sparse-Attention actions of a joint layer: the selection that a run makes and its attention under it, each against the oracle on
the queries, keys and values that the layer made, with and without lengths of prompts."""
import numpy as np
import pytest
import torch

import paper_2509_22323_amd as ra
from gpu_common import from_dev, widen
from layer_common import normal
from oracle import mask_oracle as mo
from paper_2509_22323_amd import layer as layer_module
from test_gpu_joint import oracle_joint
from test_gpu_joint_layer import halves, make
from test_gpu_mask import DELTA, oracle_joint_mask

pytestmark = pytest.mark.gpu


def structured(**kw):
    """A layer and hidden states whose blocks of 128 tokens look at some blocks more than at others: tokens of a block share a
    direction, the blocks of a pair the same one, and keys are projected as queries are."""
    layer, hidden, cond = make(image=1024, text=154, rotate=False, **kw)
    C = layer.H * layer.D
    for w in layer.weights:
        w["qkv_w"][C:2 * C] = w["qkv_w"][:C]
        w["k_norm"].copy_(w["q_norm"])
    directions = normal((layer.B, 8, C), 91, 1.5)
    for b in range(layer.B):
        for i in range(8):
            hidden[b, 128 * i:128 * (i + 1)] += directions[b, i // 2]
    return layer, hidden, cond


@pytest.mark.parametrize("kw", [dict(seed=21), dict(D=128, H=2, B=1, F=304, seed=22)], ids=str)
@pytest.mark.parametrize("lens", [None, 60], ids=["all tokens", "shorter prompts"])
@pytest.mark.parametrize("a_sparse", [1, 2, 3])
def test_sparse_actions(kw, lens, a_sparse, monkeypatch):
    layer, hidden, cond = structured(**kw)
    B, H, D, (image, text) = layer.B, layer.H, layer.D, layer.tokens
    N, nb = image + text, -(-(image + text) // 128)
    valid = np.array([N - (lens or 0) * (b + 1) // B for b in range(B)], np.int32)
    kv_lens = None if lens is None else torch.from_numpy(valid).cuda()
    start, seen = hidden.clone(), []

    def select(segments, block, **args):
        mask = torch.full((B, H, nb, nb), 9, dtype=torch.uint8, device="cuda")
        outs = real(segments, block, mask_out=mask, **args)
        joint = [np.concatenate([from_dev(seg[i]) for seg in segments], 2) for i in range(4)]
        seen.append((block, args, mask.cpu().numpy(), joint))
        return outs

    real = ra.rapid_attn_joint_select
    monkeypatch.setattr(layer_module._b, "rapid_attn_joint_select", select)
    layer.run(*halves(layer, hidden), cond, a_sparse, kv_lens)
    (block, args, mask, (q, k, v, o)), = seen
    tau = mo.LEVEL_TAU[a_sparse]
    assert block == 128 and args["text_start"] == image and abs(args["tau"] - tau) < 1e-6 and args["kv_lens"] is kv_lens
    lo, hi = (oracle_joint_mask(q, k, 128, valid, image, t) for t in (tau - DELTA, tau + DELTA))
    assert (lo <= mask).all() and (mask <= hi).all(), ((lo > mask).sum(), (mask > hi).sum())
    assert mask[:, :, :8, :8].mean() < 0.9                                         # it leaves blocks out
    for b in range(B):
        n = int(valid[b])
        want = oracle_joint(q[b:b + 1], k[b:b + 1], v[b:b + 1], n, mask[b:b + 1], 128)[0]
        got = widen(o[b])
        assert np.isfinite(got).all()
        # P and O are rounded to bf16 (2^-9 each in the mean square, relative): 2.3e-3 of the output's norm, twice that for 64 rows of a head
        for h in range(H):
            for r in range(0, n, 64):
                d, w = got[h, r:min(r + 64, n)] - want[h, r:min(r + 64, n)], want[h, r:min(r + 64, n)]
                assert np.sqrt((d * d).sum() / (w * w).sum()) <= 5e-3, (b, h, r)
    dense = start.clone()
    layer.run(*halves(layer, dense), cond, 0, kv_lens)
    hidden_lens = [slice(0, int(n)) for n in valid]
    assert all(not torch.equal(hidden[b, s], dense[b, s]) for b, s in enumerate(hidden_lens))
    again = start.clone()
    monkeypatch.setattr(layer_module._b, "rapid_attn_joint_select", real)
    layer.run(*halves(layer, again), cond, a_sparse, kv_lens)
    assert all(torch.equal(hidden[b, s], again[b, s]) for b, s in enumerate(hidden_lens))


def test_actions_leave_out_more_and_more(monkeypatch):
    layer, hidden, cond = structured(seed=23)
    start, kept = hidden.clone(), []

    def select(segments, block, **args):
        mask = torch.empty((layer.B, layer.H, 10, 10), dtype=torch.uint8, device="cuda")
        outs = real(segments, block, mask_out=mask, **args)
        kept.append(mask.cpu().numpy())
        return outs

    real = ra.rapid_attn_joint_select
    monkeypatch.setattr(layer_module._b, "rapid_attn_joint_select", select)
    for a_sparse in (1, 2, 3):
        hidden.copy_(start)
        layer.run(*halves(layer, hidden), cond, a_sparse)
    assert all((b <= a).all() for a, b in zip(kept, kept[1:])) and kept[2].sum() < kept[0].sum()
