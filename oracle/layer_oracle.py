"""Oracle for what a layer does around its attention: linear layers with their epilogue, the norm under the conditioning, the norm
and rotation of queries and keys, and the table of the rotation.

TEST INFRASTRUCTURE ONLY (imported by tests, never by the product package, and it imports nothing from it).  Everything in fp64,
from the definitions; inputs are arrays of numbers (bf16 values widened by the caller), results are not rounded.
"""
from __future__ import annotations

import math

import numpy as np


def activation(z, kind):
    if kind == "none":
        return z
    if kind == "silu":
        return z / (1.0 + np.exp(-z))
    return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))


def linear(x, w, bias=None, act="none", gate=None, residual=None):
    """x [B,n,K], w [N,K], bias [N], gate [B,N], residual [B,n,N] -> [B,n,N]"""
    z = np.matmul(x, w.T)
    if bias is not None:
        z = z + bias
    z = activation(z, act)
    if gate is not None:
        z = z * gate[:, None]
    return z if residual is None else z + residual


def norm_modulate(x, scale=None, shift=None, eps=1e-6):
    """x [B,n,C], scale and shift [B,C]"""
    d = x - x.mean(-1, keepdims=True)
    y = d / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    return y if scale is None else y * (1.0 + scale[:, None]) + shift[:, None]


def frequencies(dim, theta, scaling="none", factor=1.0, original_length=0.0, beta_fast=32.0, beta_slow=1.0):
    if scaling == "ntk":
        theta = theta * factor ** (dim / (dim - 2.0))
    f = theta ** (-2.0 * np.arange(dim // 2) / dim)
    if scaling == "linear":
        return f / factor
    if scaling == "by_parts":
        g = np.clip((original_length * f / (2.0 * math.pi) - beta_slow) / (beta_fast - beta_slow), 0.0, 1.0)
        return f * (g + (1.0 - g) / factor)
    return f


def table(positions, axes, magnitude=1.0):
    """positions [..., axes] whole numbers; axes: a dict of the arguments of frequencies for each -> [..., pairs, 2].  Angles in
    the longest floating type there is."""
    a = np.concatenate([positions[..., i, None].astype(np.longdouble) * frequencies(**x).astype(np.longdouble)
                        for i, x in enumerate(axes)], -1)
    return (magnitude * np.stack([np.cos(a), np.sin(a)], -1)).astype(np.float64)


def rotate(v, table, layout):
    """v [B,H,n,D], table [n,pairs,2] or [B,n,pairs,2]"""
    rot = 2 * table.shape[-2]
    t = table if table.ndim == 3 else table[:, None]
    c, s = t[..., 0], t[..., 1]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if layout == "interleaved" else (slice(0, rot // 2), slice(rot // 2, rot))
    y = v.copy()
    y[..., a] = v[..., a] * c - v[..., b] * s
    y[..., b] = v[..., b] * c + v[..., a] * s
    return y


def head_norm(u, weight=None, eps=1e-6):
    v = u / np.sqrt((u * u).mean(-1, keepdims=True) + eps)
    return v if weight is None else v * weight
