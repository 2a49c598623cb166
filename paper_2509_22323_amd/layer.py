"""One joint layer of an MM-DiT on the library's operators (Sec. 3.1: image and text tokens in tensors of their own, each with
weights of its own, joined for attention alone; every projection under the conditioning of the time step).

Weights are the caller's (there are none here); buffers are made once, a run allocates nothing and can be captured into a graph.
Inference only: runs are not recorded by autograd, whatever the weights require.
Runs of one layer, graphs of them included, share its buffers: they follow each other, on the stream that it was made on or behind it.
"""
from __future__ import annotations

from . import binding as _b

# of a stream: [out, in] and [out]; C = H*D hidden channels, F of the feed-forward block
WEIGHTS = ("mod_w", "mod_b",           # [6C, C]: shift, scale, gate of the attention block, shift, scale, gate of the feed-forward block
           "qkv_w", "qkv_b",           # [3C, C]: queries, keys, values, each head after head
           "q_norm", "k_norm",         # [D], or None
           "out_w", "out_b",           # [C, C]
           "ff_in_w", "ff_in_b",       # [F, C]
           "ff_out_w", "ff_out_b")     # [C, F]


_NONE_ALLOWED = ("mod_b", "qkv_b", "q_norm", "k_norm", "out_b", "ff_in_b", "ff_out_b")


def _check_sizes(weights, B, H, D, image, text, layout, eps):
    """What a run would refuse half way through it."""
    if B < 1 or H < 1 or D not in (64, 128):
        raise ValueError(f"B = {B}, H = {H}, D = {D}: D is 64 or 128, B and H are at least 1")
    if image < 128 or image % 128 != 0:
        raise ValueError(f"{image} image tokens: their number must be a multiple of 128")
    if text < 1:
        raise ValueError(f"{text} text tokens: there must be one at least")
    if layout not in _b.ROPE_LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(_b.ROPE_LAYOUTS)}")
    if not eps >= 0:
        raise ValueError("eps must not be negative")
    if len(weights) != 2:
        raise ValueError("weights: of the image stream and of the text stream")
    C = H * D
    for stream, w in zip(("image", "text"), weights):
        F = w["ff_in_w"].shape[0]
        if F < 8 or F % 8 != 0:
            raise ValueError(f"{stream} stream: {F} channels of the feed-forward block, not a multiple of 8")
        for name, shape in zip(WEIGHTS, ((6 * C, C), (6 * C,), (3 * C, C), (3 * C,), (D,), (D,), (C, C), (C,), (F, C), (F,), (C, F), (C,))):
            if w[name] is None and name in _NONE_ALLOWED:
                continue
            if w[name] is None or tuple(w[name].shape) != shape:
                raise ValueError(f"{stream} stream: {name} must be {list(shape)}, not {None if w[name] is None else list(w[name].shape)}")


class JointLayer:
    """weights: (of the image stream, of the text stream), each a dict of CUDA bf16 tensors named as in WEIGHTS (biases and norms
    may be None).  positions (CUDA int32 [image + text, axes], or [B, image + text, axes]) and axes (RopeAxis each): the rotation
    of queries and keys; None = none.  image is a multiple of 128, F of 8."""

    def __init__(self, weights, B, H, D, image, text, positions=None, axes=None, layout="interleaved", eps=1e-6):
        import torch
        _check_sizes(weights, B, H, D, image, text, layout, eps)
        self.weights, self.B, self.H, self.D, self.layout, self.eps = weights, B, H, D, layout, eps
        self.tokens = (image, text)
        device = weights[0]["qkv_w"].device
        self.device = device.index
        C, wide = H * D, [w["ff_in_w"].shape[0] for w in weights]

        def empty(*shape, dtype=torch.bfloat16):
            return torch.empty(shape, dtype=dtype, device=device)

        self.mod = [empty(B, 6, C) for _ in weights]
        self.h = [empty(B, n, C) for n in self.tokens]
        self.qkv = [empty(B, n, 3, H, D) for n in self.tokens]
        self.o = [empty(B, n, H, D) for n in self.tokens]
        self.f = [empty(B, n, F) for n, F in zip(self.tokens, wide)]
        self.table = None
        if positions is not None:
            if tuple(positions.shape) not in ((image + text, len(axes)), (B, image + text, len(axes))):
                raise ValueError(f"positions must be [{image + text}, {len(axes)}] or [{B}, {image + text}, {len(axes)}], not {list(positions.shape)}")
            self.table = empty(*positions.shape[:-1], sum(int(a.dim) for a in axes) // 2, 2, dtype=torch.float32)
            _b.rapid_rope_table(positions, axes, self.table)
        need = max(_b.rapid_linear_workspace_bytes(M, N, K) for n, F in zip(self.tokens, wide)
                   for M, N, K in ((B, 6 * C, C), (B * n, 3 * C, C), (B * n, C, C), (B * n, F, C), (B * n, C, F)))
        self.workspace = empty(max(need, 16), dtype=torch.uint8)
        self.select_workspace = empty(max(_b.rapid_attn_joint_select_workspace_bytes(B, H, image + text, D, 128), 16),
                                      dtype=torch.uint8)
        self.rows = [tuple(t.permute(2, 0, 3, 1, 4)) for t in self.qkv]            # (q, k, v) [B, H, n, D] of each stream
        self.norms = [(w["q_norm"], w["k_norm"]) for w in weights]

    def run(self, image, text, conditioning, a_sparse=0, kv_lens=None):
        """image [B, n, C], text [B, m, C] <- the layer's output, in place.  conditioning: [B, C], the vector that every layer's
        projection takes (its activation done); a_sparse: the Sparse-Attention action (0: dense); kv_lens as rapid_attn_joint."""
        if int(a_sparse) not in range(4):
            raise ValueError(f"a_sparse = {a_sparse}: the Sparse-Attention actions are 0 to 3")
        import torch
        if torch._C._cuda_getDevice() == self.device:
            return self._run(image, text, conditioning, a_sparse, kv_lens)
        with torch.cuda.device(self.device):               # (the attention calls launch on the current device)
            return self._run(image, text, conditioning, a_sparse, kv_lens)

    def _run(self, image, text, conditioning, a_sparse, kv_lens):
        hidden = (image, text)
        for x, h, mod, qkv, w in zip(hidden, self.h, self.mod, self.qkv, self.weights):
            _b.rapid_linear(conditioning, w["mod_w"], mod.view(self.B, -1), w["mod_b"], workspace=self.workspace)
            _b.rapid_norm_modulate(x, h, mod[:, 1], mod[:, 0], self.eps)
            _b.rapid_linear(h, w["qkv_w"], qkv.view(*h.shape[:2], -1), w["qkv_b"], workspace=self.workspace)
        _b.rapid_qk_norm_rope([(q, k, q, k) for q, k, _ in self.rows], self.norms, self.table, self.layout, self.eps)
        segments = [(q, k, v, o.transpose(1, 2)) for (q, k, v), o in zip(self.rows, self.o)]
        if a_sparse == 0:
            _b.rapid_attn_joint(segments, kv_lens=kv_lens)
        else:
            _b.rapid_attn_joint_select(segments, 128, kv_lens=kv_lens, text_start=self.tokens[0],
                                       tau=_b.rapid_mask_level_tau(a_sparse), workspace=self.select_workspace)
        for x, h, mod, o, f, w in zip(hidden, self.h, self.mod, self.o, self.f, self.weights):
            _b.rapid_linear(o.view(h.shape), w["out_w"], x, w["out_b"], "none", mod[:, 2], x, self.workspace)
            _b.rapid_norm_modulate(x, h, mod[:, 4], mod[:, 3], self.eps)
            _b.rapid_linear(h, w["ff_in_w"], f, w["ff_in_b"], "gelu_tanh", workspace=self.workspace)
            _b.rapid_linear(f, w["ff_out_w"], x, w["ff_out_b"], "none", mod[:, 5], x, self.workspace)
        return image, text
