"""Helpers of the tests of the operators around the attention: tensors in the middle of larger buffers of NaN, and error bounds."""
import numpy as np
import torch

BF16_STEP = 2.0 ** -8          # half a step of bf16, relative to the value
NAN = float("nan")


def widen(t):
    return t.double().cpu().numpy()


def normal(shape, seed, scale=1.0, mean=0.0):
    """bf16 on the GPU, from the seed alone"""
    rng = np.random.default_rng(seed)
    return torch.from_numpy((rng.standard_normal(shape) * scale + mean).astype(np.float32)).to(torch.bfloat16).cuda()


def inside(t, before, after, pad_last=0):
    """The values of t [B, n, width] as a slice of a NaN-filled [B, before + n + after, width + pad_last] buffer: (view, buffer)"""
    B, n, width = t.shape
    big = torch.full((B, before + n + after, width + pad_last), NAN, dtype=t.dtype, device=t.device)
    view = big[:, before:before + n, :width]
    view.copy_(t)
    return view, big


def untouched_around(view, big):
    """Everything of the NaN-filled buffer but the view is NaN still."""
    keep = torch.ones_like(big, dtype=torch.bool)
    keep.as_strided(view.shape, view.stride(), view.storage_offset() - big.storage_offset())[...] = False
    return bool(torch.isnan(big[keep]).all())


def assert_within(got, want, bound, what=""):
    got, bound = widen(got), np.broadcast_to(bound, want.shape)
    assert np.isfinite(got).all(), f"{what}: not finite"
    over = np.abs(got - want) - bound
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, f"{what}: {got[at]} for {want[at]} at {at}, bound {bound[at]:.3e}; {(over > 0).sum()} of {over.size} beyond"
