"""The operators of a layer around its joint attention, as cases to time: the linear layers with their epilogue,
the norm under the conditioning's shift and scale, the norm of every head's queries and keys with the rotation by
position, the rotation alone, and the table of angles that both read.

Widths are those of the models that `workloads/` stands for (24 heads of 64 or 128, 4096 image tokens and up to
512 text tokens at 1024 x 1024) and of the larger 64-wide one of `perf/cases.py` (38 heads).  `run` computes an
operator in elementary torch operations in 32 bits (angles in 64), or by this package where `own` is set.
Everything a program keeps between calls (weights, tables, outputs, workspaces) is made in `prepare`.
"""
import math

import torch

own = False                                            # True: `run` calls this package's operators

LARGEST = 2.0 * 8192 * 2432 * 9728                     # multiply-adds of the largest listed case, twice


def listed():
    return [
        # the conditioning of a layer: one row a sample, six vectors out; a guidance pair.  Latency, and 28 MB of weights
        dict(name="linear_modulation", kind="linear", B=2, n=1, K=1536, N=9216, act="none", gate=False, residual=False, bias=True),
        # queries, keys and values of the image stream, 1024 x 1024, guidance pair
        dict(name="linear_qkv_image", kind="linear", B=2, n=4096, K=1536, N=4608, act="none", gate=False, residual=False, bias=True),
        # first half of the text stream's feed-forward block: 333 tokens a sample (an odd number), wide output
        dict(name="linear_ff_in_text", kind="linear", B=2, n=333, K=2432, N=9728, act="gelu_tanh", gate=False, residual=False, bias=True),
        # second half of the image stream's feed-forward block, gated onto the residual stream: the largest
        dict(name="linear_ff_out_image", kind="linear", B=2, n=4096, K=9728, N=2432, act="none", gate=True, residual=True, bias=True),
        # norm before the attention, a rollout group of eight samples at 1024 x 1024
        dict(name="modulate_group", kind="modulate", B=8, n=4096, C=1536, affine=True),
        # the text stream of one sample
        dict(name="modulate_text", kind="modulate", B=1, n=333, C=2432, affine=True),
        # queries and keys of image and text as the fused projections hold them, 128-wide heads, three position axes
        dict(name="qk_norm_rope_flux_1024", kind="qk", B=1, H=24, image=4096, text=512, D=128, rot=128, layout="interleaved", fused=True),
        # norm alone (a model without rotation), 512 x 512, guidance pair, odd text length
        dict(name="qk_norm_sd3_512", kind="qk", B=2, H=24, image=1024, text=333, D=64, rot=0, layout="interleaved", fused=True),
        # the smallest rotation of the test workloads, a part of the head in two halves: latency
        dict(name="rope_tiny", kind="rope", B=1, H=2, image=256, text=0, D=64, rot=32, layout="half", fused=False),
        # a 2048 x 2048 image, head-major tensors
        dict(name="rope_flux_2048", kind="rope", B=1, H=24, image=16384, text=512, D=128, rot=128, layout="interleaved", fused=False),
        # angles of 1024 x 1024 image and text tokens over three axes
        dict(name="table_flux_1024", kind="table", B=1, side=64, text=512, dims="16,56,56", scaling="none", factor=1.0),
        # angles of a group of images four times as wide as those trained on, frequencies scaled by parts
        dict(name="table_4096_group", kind="table", B=4, side=256, text=512, dims="16,56,56", scaling="by_parts", factor=4.0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "linear", "modulate", "qk", "qk", "rope", "table"])
    B = _log_uniform(rng, 1, 8)
    if kind == "linear":
        n = 1 if rng.random() < 0.2 else _log_uniform(rng, 1, 16384)
        return dict(kind=kind, B=B, n=n, K=8 * _log_uniform(rng, 8, 1216), N=_log_uniform(rng, 16, 9728),
                    act=rng.choice(["none", "silu", "gelu_tanh"]), gate=rng.random() < 0.4, residual=rng.random() < 0.5,
                    bias=rng.random() < 0.8)
    if kind == "modulate":
        return dict(kind=kind, B=B, n=_log_uniform(rng, 1, 16384), C=8 * _log_uniform(rng, 8, 1216), affine=rng.random() < 0.9)
    if kind == "table":
        dims = rng.choice(["16,56,56", "32,32", "64", "128", "8,28,28", "16,24,24"])
        return dict(kind=kind, B=B, side=_log_uniform(rng, 1, 256), text=rng.randint(1, 512), dims=dims,
                    scaling=rng.choice(["none", "linear", "ntk", "by_parts"]), factor=round(rng.uniform(1.0, 8.0), 2))
    D = rng.choice([64, 128])
    rot = rng.choice([D, D, D // 2, 16, 0] if kind == "qk" else [D, D, D // 2, 16])
    return dict(kind=kind, B=B, H=rng.choice([1, 2, 5, 8, 16, 24, 24, 38]), image=_log_uniform(rng, 1, 16384),
                text=rng.choice([0, rng.randint(1, 512)]), D=D, rot=rot, layout=rng.choice(["interleaved", "half"]),
                fused=rng.random() < 0.5)


def draw(rng):
    """A case of the same ranges: 1 to 8 samples, 1 to 16384 tokens, widths of 64 to 9728 in and 16 to 9728 (odd ones among
    them) out, both head sizes; no more work than the largest listed one and at most 1 GB read and written."""
    while True:
        case = _draw(rng)
        w = work(case)
        if w["flops"] <= LARGEST and w["bytes"] <= 1.0e9:
            return case


# ------------------------------------------------------------------------------- inputs
def _dims(case):
    return [int(d) for d in case["dims"].split(",")]


def _frequencies(dims, scaling, factor):
    """Radians per position of every pair, in 64 bits: theta 10000; trained on 64 positions an axis."""
    parts = []
    for d in dims:
        i = torch.arange(d // 2, dtype=torch.float64, device="cuda")
        theta = 10000.0 * (factor ** (d / (d - 2.0)) if scaling == "ntk" else 1.0)
        f = torch.exp(-math.log(theta) * 2.0 * i / d)
        if scaling == "linear":
            f = f / factor
        if scaling == "by_parts":
            keep = ((64.0 * f / (2.0 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
            f = f * (keep + (1.0 - keep) / factor)
        parts.append(f)
    return parts


def _positions(B, side, text, axes, scatter=0):
    """int32 [B, side^2 + text, axes]: (0, row, column) of image tokens and zeros for text with three axes, (row, column)
    with two, the token's number with one; sample b starts at (b + 1) * scatter (a crop of a larger image)."""
    t = torch.arange(side * side + text, device="cuda")
    image = t < side * side
    zero = torch.zeros_like(t)
    row, column = torch.where(image, t // side, zero), torch.where(image, t % side, zero)
    columns = {1: [t], 2: [row, column], 3: [zero, row, column]}[axes]
    p = torch.stack(columns, -1).int().expand(B, -1, -1).clone()
    return p + (torch.arange(1, B + 1, device="cuda", dtype=torch.int32) * scatter)[:, None, None]


def _normal(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


def _inputs(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    s = dict(case)
    if case["kind"] == "linear":
        B, n, K, N = case["B"], case["n"], case["K"], case["N"]
        x = torch.randn((B, n, K), generator=g, device="cuda")
        s["x"] = (x * torch.sigmoid(1.702 * x) if case["gate"] else x).to(torch.bfloat16)       # what an activation leaves, or a norm
        s["w"] = _normal(g, N, K, scale=K ** -0.5)
        s["b"] = _normal(g, N, scale=0.1) if case["bias"] else None
        # the gate is one of six vectors that the conditioning gives
        s["g"] = _normal(g, B, 6, N, scale=0.5)[:, 5] if case["gate"] else None
        s["r"] = _normal(g, B, n, N) if case["residual"] else None
        s["out"] = torch.empty((B, n, N), device="cuda", dtype=torch.bfloat16)
    elif case["kind"] == "modulate":
        B, n, C = case["B"], case["n"], case["C"]
        s["x"] = _normal(g, B, n, C, scale=3.0) + _normal(g, 1, 1, C)          # channels of different mean, as hidden states have
        vectors = _normal(g, B, 6, C, scale=0.3)
        s["shift"], s["scale"] = (vectors[:, 0], vectors[:, 1]) if case["affine"] else (None, None)
        s["out"] = torch.empty_like(s["x"])
    elif case["kind"] == "table":
        s["positions"] = _positions(case["B"], case["side"], case["text"], len(_dims(case)), 1 + seed % 1000)
        s["out"] = torch.empty((case["B"], case["side"] ** 2 + case["text"], sum(_dims(case)) // 2, 2), device="cuda")
    else:
        B, H, D, rot = case["B"], case["H"], case["D"], case["rot"]
        s["segments"], s["weights"] = [], []
        for n in (case["image"], case["text"]):
            if n == 0:
                continue
            if case["fused"]:                                                  # as a fused projection holds them, and as it would again
                t = _normal(g, B, n, 3, H, D, scale=2.0).permute(2, 0, 3, 1, 4)
                o = torch.empty((2, B, n, H, D), device="cuda", dtype=torch.bfloat16).permute(0, 1, 3, 2, 4)
            else:
                t = _normal(g, 2, B, H, n, D, scale=2.0)
                o = torch.empty_like(t)
            s["segments"].append((t[0], t[1], o[0], o[1]))
            s["weights"].append(tuple((1.0 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2)))
        s["table"] = None
        if rot:
            side = math.isqrt(case["image"])
            dims = {16: (16,), 32: (32,), 64: (32, 32), 128: (16, 56, 56)}[rot]
            tokens = case["image"] + case["text"]
            p = _positions(1, side, tokens - side * side, len(dims), 0)[0].double()
            a = torch.cat([p[:, i, None] * f for i, f in enumerate(_frequencies(dims, "none", 1.0))], -1)
            s["table"] = torch.stack([a.cos(), a.sin()], -1).float()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and case["kind"] == "linear":
        import paper_2509_22323_amd as ra
        bytes_ = ra.rapid_linear_workspace_bytes(case["B"] * case["n"], case["N"], case["K"])
        s["workspace"] = torch.empty(max(bytes_, 16), dtype=torch.uint8, device="cuda")
    if own and case["kind"] == "table":
        import paper_2509_22323_amd as ra
        s["axes"] = [ra.RopeAxis(d, 10000.0, case["scaling"], case["factor"], 64.0) for d in _dims(case)]
    return s


# ------------------------------------------------------------------------------- one pass
def _own(s):
    import paper_2509_22323_amd as ra
    if s["kind"] == "linear":
        return ra.rapid_linear(s["x"], s["w"], s["out"], s["b"], s["act"], s["g"], s["r"], s["workspace"])
    if s["kind"] == "modulate":
        return ra.rapid_norm_modulate(s["x"], s["out"], s["scale"], s["shift"])
    if s["kind"] == "table":
        return ra.rapid_rope_table(s["positions"], s["axes"], s["out"])
    if s["kind"] == "rope":
        return ra.rapid_rope(s["segments"], s["table"], s["layout"])
    return ra.rapid_qk_norm_rope(s["segments"], s["weights"], s["table"], s["layout"])


def _rotate(x, table, layout):
    """x fp32 [B, H, n, D], table [n, rot / 2, 2]"""
    rot = 2 * table.shape[1]
    c, s = table[..., 0], table[..., 1]
    if layout == "interleaved":
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def run(s):
    if own:
        return _own(s)
    if s["kind"] == "linear":
        B, n, K = s["x"].shape
        y = s["x"].float().reshape(B * n, K) @ s["w"].float().t()
        if s["b"] is not None:
            y = y + s["b"].float()
        if s["act"] == "silu":
            y = y / (1.0 + torch.exp(-y))
        if s["act"] == "gelu_tanh":
            y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
        y = y.reshape(B, n, -1)
        if s["g"] is not None:
            y = y * s["g"].float()[:, None]
        if s["r"] is not None:
            y = y + s["r"].float()
        return y.to(torch.bfloat16)
    if s["kind"] == "modulate":
        x = s["x"].float()
        x = x - x.mean(-1, keepdim=True)
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        if s["scale"] is not None:
            y = y * (1.0 + s["scale"].float()[:, None]) + s["shift"].float()[:, None]
        return y.to(torch.bfloat16)
    if s["kind"] == "table":
        p = s["positions"].double()
        a = torch.cat([p[..., i, None] * f for i, f in enumerate(_frequencies(_dims(s), s["scaling"], s["factor"]))], -1)
        return torch.stack([a.cos(), a.sin()], -1).float()
    made, first = [], 0
    for i, (q, k, _, _) in enumerate(s["segments"]):
        for j, t in enumerate((q, k)):
            x = t.float()
            if s["kind"] == "qk":
                x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * s["weights"][i][j].float()
            if s["table"] is not None:
                x = _rotate(x, s["table"][first:first + t.shape[2]], s["layout"])
            made.append(x.to(torch.bfloat16))
        first += q.shape[2]
    return made


# ------------------------------------------------------------------------------- bounds and exact values
def work(case):
    if case["kind"] == "linear":
        M, K, N = case["B"] * case["n"], case["K"], case["N"]
        elements = M * K + N * K + M * N * (2 if case["residual"] else 1) + (N if case["bias"] else 0) + (case["B"] * N if case["gate"] else 0)
        return {"bytes": 2.0 * elements, "flops": 2.0 * M * K * N}
    if case["kind"] == "modulate":
        elements = case["B"] * case["n"] * case["C"]
        return {"bytes": 4.0 * elements + (4.0 * case["B"] * case["C"] if case["affine"] else 0.0), "flops": 8.0 * elements}
    if case["kind"] == "table":
        tokens, half = case["B"] * (case["side"] ** 2 + case["text"]), sum(_dims(case)) // 2
        return {"bytes": tokens * (4.0 * len(_dims(case)) + 8.0 * half), "flops": 50.0 * tokens * half}
    tokens = case["image"] + case["text"]
    elements = 2.0 * case["B"] * case["H"] * tokens * case["D"]
    return {"bytes": 4.0 * elements + 4.0 * tokens * case["rot"], "flops": (4.0 if case["kind"] == "qk" else 0.0) * elements
            + 3.0 * elements * case["rot"] / case["D"]}


def _exact_turn(x, angle_cos, angle_sin, layout):
    """Every pair as a complex number times cos + i sin."""
    rot = 2 * angle_cos.shape[-1]
    turn = torch.complex(angle_cos, angle_sin)
    pairs = x[..., :rot].unflatten(-1, (rot // 2, 2)) if layout == "interleaved" else x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    turned = z.flatten(-2) if layout == "interleaved" else z.transpose(-1, -2).flatten(-2)
    y = x.clone()
    y[..., :rot] = turned
    return y


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "linear":
        B, n, K = s["x"].shape
        y = torch.mm(s["x"].double().view(B * n, K), s["w"].double().t().contiguous()).view(B, n, case["N"])
        if case["bias"]:
            y.add_(s["b"].double())
        if case["act"] == "silu":
            y.mul_(torch.sigmoid(y))
        elif case["act"] == "gelu_tanh":
            y.mul_(torch.sigmoid(math.sqrt(8.0 / math.pi) * (y + 0.044715 * y.pow(3))))
        if case["gate"]:
            y.mul_(s["g"].double().unsqueeze(1))
        if case["residual"]:
            y.add_(s["r"].double())
        return y
    if case["kind"] == "modulate":
        x = s["x"].double()
        variance, mean = torch.var_mean(x, dim=-1, correction=0, keepdim=True)
        y = (x - mean) / (variance + 1e-6).sqrt()
        if case["affine"]:
            y = torch.addcmul(s["shift"].double().unsqueeze(1), y, 1.0 + s["scale"].double().unsqueeze(1))
        return y
    if case["kind"] == "table":
        a = []
        for axis, d in enumerate(_dims(case)):
            for pair in range(d // 2):
                theta, factor = 10000.0, case["factor"]
                if case["scaling"] == "ntk":
                    theta *= factor ** (d / (d - 2))
                f = theta ** (-2 * pair / d)
                if case["scaling"] == "linear":
                    f /= factor
                if case["scaling"] == "by_parts":
                    turns = 64.0 * f / (2 * math.pi)                           # over the positions trained on
                    keep = min(max((turns - 1.0) / 31.0, 0.0), 1.0)
                    f = keep * f + (1.0 - keep) * f / factor
                a.append(s["positions"][..., axis].double() * f)
        a = torch.stack(a, -1)
        return torch.stack([torch.cos(a), torch.sin(a)], -1)
    made, first = [], 0
    for (q, k, _, _), weights in zip(s["segments"], s["weights"]):
        for t, weight in zip((q, k), weights):
            x = t.double()
            if case["kind"] == "qk":
                x = x / (x.square().sum(-1, keepdim=True) / case["D"] + 1e-6).sqrt() * weight.double()
            if s["table"] is not None:
                rows = s["table"][first:first + t.shape[2]].double()
                x = _exact_turn(x, rows[..., 0], rows[..., 1], case["layout"])
            made.append(x)
        first += q.shape[2]
    return made
