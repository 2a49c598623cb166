"""Oracle for layers in 8 bits over packed sequences: rows as 8-bit integers, the norm that ends in them, linear layers on them, and
the attention of packed documents.

TEST INFRASTRUCTURE ONLY (imported by tests, never by the product package, and it imports nothing from it).  Everything in fp64,
from the definitions; inputs are arrays of numbers (bf16 values widened by the caller), results are not rounded but where the
definition rounds.
"""
from __future__ import annotations

import numpy as np

from . import layer_oracle as lo


def quantize(x):
    """x [..., K] -> (whole numbers [..., K], scale [...]): round(127 x / m), ties to even, and m / 127.  127 x is exact and the
    quotient rounded once, so for x of few bits (bf16) a tie is one only where the exact quotient is."""
    m = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1)
    plain = ~bad & (m > 0)
    some = np.where(plain, m, 1.0)[..., None]
    q = np.where(plain[..., None], np.rint(127.0 * np.where(plain[..., None], x, 0.0) / some), 0.0)
    return q, np.where(bad, np.nan, m / 127.0)


def norm_modulate(x, scale=None, shift=None, eps=1e-6, document=None):
    """x [B,n,C]; scale, shift [B,C], or [documents,C] with document [B,n] (rows of no document: those of document 0)"""
    y = lo.norm_modulate(x, None, None, eps)
    if scale is None:
        return y
    if document is None:
        return y * (1.0 + scale[:, None]) + shift[:, None]
    return y * (1.0 + scale[document.clip(0)]) + shift[document.clip(0)]


def linear(x, x_scale, w, w_scale, bias=None, act="none", gate=None, residual=None, document=None):
    """x [B,n,K] and w [N,K] whole numbers, x_scale [B,n], w_scale [N]; gate [B,N], or [documents,N] with document [B,n]"""
    z = np.matmul(x, w.T) * x_scale[..., None] * w_scale
    if bias is not None:
        z = z + bias
    z = lo.activation(z, act)
    if gate is not None:
        z = z * (gate[:, None] if document is None else gate[document.clip(0)])
    return z if residual is None else z + residual


def visible(document, order=None):
    """[B,N,N]: whether query i sees key j"""
    s = (document[:, :, None] == document[:, None, :]) & (document >= 0)[:, None, :]
    return s if order is None else s & (order[:, None, :] <= order[:, :, None])


def attention(q, k, v, document, order=None, cap=0.0, scale=None):
    """q, k, v [B,H,N,D], document and order [B,N] -> (o [B,H,N,D], the softmax [B,H,N,N]).  What is not visible has no part in a
    sum, whatever it holds."""
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    see = visible(document, order)[:, None]
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.matmul(q, np.swapaxes(k, -1, -2)) * scale
        if cap:
            s = cap * np.tanh(s / cap)
        s = np.where(see, s, -np.inf)
        top = s.max(-1, keepdims=True)
        p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
        p = np.where(see, p, 0.0)
        l = p.sum(-1, keepdims=True)
        p = p / np.where(l > 0, l, 1.0)
        if np.isfinite(v).all():
            return np.matmul(p, v), p
        o = np.zeros(q.shape)
        for b, h, i in np.ndindex(*q.shape[:3]):
            keys = see[b, 0, i]
            o[b, h, i] = (p[b, h, i, keys][:, None] * v[b, h, keys]).sum(0)
        return o, p
