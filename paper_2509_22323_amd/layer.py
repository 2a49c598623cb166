"""One joint layer of an MM-DiT on the library's operators (Sec. 3.1: image and text tokens in tensors of their own, each with
weights of its own, joined for attention alone; every projection under the conditioning of the time step): in bf16 over a batch, or in
8 bits over requests of any sizes packed into one sequence.

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


MOST = (2 - 2.0 ** -23) * 2.0 ** 127   # of fp32
_NONE_ALLOWED = ("mod_b", "qkv_b", "q_norm", "k_norm", "out_b", "ff_in_b", "ff_out_b")


def _check_sizes(weights, B, H, D, image, text, layout, eps, tile=128, wide=8):
    """What a run would refuse half way through it."""
    if B < 1 or H < 1 or D not in (64, 128):
        raise ValueError(f"B = {B}, H = {H}, D = {D}: D is 64 or 128, B and H are at least 1")
    if image < tile or image % tile != 0:
        raise ValueError(f"{image} image tokens: their number must be a multiple of {tile}")
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
        if F < wide or F % wide != 0:
            raise ValueError(f"{stream} stream: {F} channels of the feed-forward block, not a multiple of {wide}")
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


class PackedLayer:
    """The same layer in 8 bits over packed requests: the image tokens of all of them one after the other in one tensor, their texts in
    another, each request (a document) under a conditioning vector of its own and seeing itself alone.  The projections are products of
    8-bit integers with scales for each token and channel, and those of the conditioning, in bf16, are made of up to four requests at a
    time, whose sums are each request's own; what a token comes to does not depend on what it is packed with, but for the order in
    which its attention's sums are added.

    weights as JointLayer takes them; those of the projections are quantised here, on the current stream, and not kept: a run on
    another stream has to wait for that one first, as with any tensor.  Its buffers serve one run at a time.  image, text: tokens that the
    tensors of a run have, any numbers; documents: how many requests a run holds at most; axes (RopeAxis each): the rotation of
    queries and keys, None = none.  F is a multiple of 16."""

    PRODUCTS = ("qkv_w", "out_w", "ff_in_w", "ff_out_w")
    # Rows of a product in bf16 that are each by itself (of more, sums are added in another order for other numbers of them)
    ROWS = 4

    def __init__(self, weights, H, D, image, text, documents, axes=None, layout="interleaved", eps=1e-6):
        import torch
        _check_sizes(weights, 1, H, D, image, text, layout, eps, 1, 16)
        if documents < 1:
            raise ValueError(f"{documents} documents: there must be one at least")
        if not eps <= MOST:
            raise ValueError("eps must be finite in fp32")
        if H * D > 16384:
            raise ValueError(f"{H * D} channels: a norm has 16384 at most")
        for stream, w in zip(("image", "text"), weights):
            if w["ff_in_w"].shape[0] > 2 ** 17 - 16:
                raise ValueError(f"{stream} stream: {w['ff_in_w'].shape[0]} channels of the feed-forward block, of which a product in 8 bits takes 2^17 - 16 at most")
        self.H, self.D, self.layout, self.eps, self.axes, self.documents = H, D, layout, eps, axes, documents
        self.tokens = (image, text)
        self.small = [{k: t for k, t in w.items() if k not in self.PRODUCTS} for w in weights]
        device = weights[0]["qkv_w"].device
        self.device = device.index
        C, wide = H * D, [w["ff_in_w"].shape[0] for w in weights]

        def empty(*shape, dtype=torch.bfloat16):
            return torch.empty(shape, dtype=dtype, device=device)

        def rows(n, width):                                # 8-bit rows and their scales (zeros: rows of no document stay as they are)
            return torch.zeros((n, width), dtype=torch.int8, device=device), torch.zeros(n, dtype=torch.float32, device=device)

        self.weights = [{k: _b.rapid_quantize_rows(w[k], empty(*w[k].shape, dtype=torch.int8), empty(w[k].shape[0], dtype=torch.float32))
                         for k in self.PRODUCTS} for w in weights]
        self.mod = [empty(documents, 6, C) for _ in weights]
        self.h = [rows(n, C) for n in self.tokens]
        self.qkv = [empty(1, n, 3, H, D) for n in self.tokens]
        self.o = [empty(1, n, H, D) for n in self.tokens]
        self.o8 = [rows(n, C) for n in self.tokens]
        self.f = [empty(n, F) for n, F in zip(self.tokens, wide)]
        self.f8 = [rows(n, F) for n, F in zip(self.tokens, wide)]
        self.table = None if axes is None else empty(image + text, sum(int(a.dim) for a in axes) // 2, 2, dtype=torch.float32)
        need = max(_b.rapid_linear_int8_workspace_bytes(M, N, K) for n, F in zip(self.tokens, wide)
                   for M, N, K in ((n, 3 * C, C), (n, C, C), (n, F, C), (n, C, F)))
        self.workspace = empty(max(need, 16), dtype=torch.uint8)
        self.attention_workspace = empty(max(_b.rapid_attn_packed_workspace_bytes(1, H, image + text, D), 16), dtype=torch.uint8)
        self.rows = [tuple(t.permute(2, 0, 3, 1, 4)) for t in self.qkv]            # (q, k, v) [1, H, n, D] of each stream
        self.norms = [(w["q_norm"], w["k_norm"]) for w in weights]

    def run(self, image, text, conditioning, document, positions=None, order=None, cap=0.0):
        """image [n, C], text [m, C] <- the layer's output, in place; rows of no document stay as they are.  conditioning: [documents, C]
        (as many as there are, at most those that the layer was made for); document: int32 [n + m], the request of every token of
        image and then text, -1 for padding; positions: int32 [n + m, axes], needed where the layer has axes; order, cap as
        rapid_attn_packed."""
        if conditioning.dim() != 2 or not 1 <= conditioning.shape[0] <= self.documents:
            raise ValueError(f"conditioning: {list(conditioning.shape)}, a vector each of 1 to {self.documents} documents")
        if (positions is None) != (self.axes is None):
            raise ValueError("positions: where the layer has axes, and only there")
        for name, t, n in zip(("image", "text"), (image, text), self.tokens):
            if tuple(t.shape) != (n, self.H * self.D) or (n > 1 and t.stride(0) < t.shape[1]):
                raise ValueError(f"{name}: rows [{n}, {self.H * self.D}] that share no element, not {list(t.shape)} with strides {list(t.stride())}")
        for name, t in (("document", document), ("order", order)):
            if t is not None and tuple(t.shape) != (sum(self.tokens),):
                raise ValueError(f"{name} must be [{sum(self.tokens)}], not {list(t.shape)}")
        if not (cap == 0 or 2.0 ** -149 <= cap <= MOST):
            raise ValueError("cap must be 0 or a positive number of fp32")
        import torch
        if torch._C._cuda_getDevice() == self.device:
            return self._run(image, text, conditioning, document, positions, order, cap)
        with torch.cuda.device(self.device):
            return self._run(image, text, conditioning, document, positions, order, cap)

    def _run(self, image, text, conditioning, document, positions, order, cap):
        hidden = (image, text)
        n = self.tokens[0]
        documents = (document[:n], document[n:])
        mods = [mod[:conditioning.shape[0]] for mod in self.mod]
        requests = conditioning.split(self.ROWS)
        if positions is not None:
            _b.rapid_rope_table(positions, self.axes, self.table)

        def linear(of, w, name, bias, out, *rest, document=None):
            _b.rapid_linear_int8(*of, *w[name], out, bias, *rest, document=document, workspace=self.workspace)

        for x, h, mod, qkv, w, small, d in zip(hidden, self.h, mods, self.qkv, self.weights, self.small, documents):
            for some, out in zip(requests, mod.view(mod.shape[0], -1).split(self.ROWS)):
                _b.rapid_linear(some, small["mod_w"], out, small["mod_b"])
            _b.rapid_norm_modulate_int8(x, *h, mod[:, 1], mod[:, 0], self.eps, d)
            linear(h, w, "qkv_w", small["qkv_b"], qkv.view(x.shape[0], -1))
        _b.rapid_qk_norm_rope([(q, k, q, k) for q, k, _ in self.rows], self.norms, self.table, self.layout, self.eps)
        _b.rapid_attn_packed([(q, k, v, o.transpose(1, 2)) for (q, k, v), o in zip(self.rows, self.o)], document, order, cap,
                             workspace=self.attention_workspace)
        for i, (x, h, mod, w, small, d) in enumerate(zip(hidden, self.h, mods, self.weights, self.small, documents)):
            _b.rapid_quantize_rows(self.o[i].view(x.shape), *self.o8[i])
            linear(self.o8[i], w, "out_w", small["out_b"], x, "none", mod[:, 2], x, document=d)
            _b.rapid_norm_modulate_int8(x, *h, mod[:, 4], mod[:, 3], self.eps, d)
            linear(h, w, "ff_in_w", small["ff_in_b"], self.f[i], "gelu_tanh")
            _b.rapid_quantize_rows(self.f[i], *self.f8[i])
            linear(self.f8[i], w, "ff_out_w", small["ff_out_b"], x, "none", mod[:, 5], x, document=d)
        return image, text
