"""Layers in 8 bits over packed sequences, as cases to time: the quantisation of rows to 8-bit integers, the norm under the
conditioning's shift and scale that ends in such rows, the linear layers as products of 8-bit integers with scales for each token and
channel, and the attention of several documents (an image with its text each) packed into one joint sequence, under an order of
their tokens and a cap on the scores.

Widths are those of `perf/operators.py` (24 heads of 64 or 128, 38 of 64; images of 1024 x 1024 and smaller, up to 512 text tokens).
`run` computes an operator in elementary torch operations in 32 bits (in 64 what ends next to a border between two integers), or by
this package where `own` is set.  Everything a program keeps between calls (weights, outputs, workspaces) is made in `prepare`.
Rows of 8-bit integers are returned as the numbers that they stand for.
"""
import math

import torch

own = False                                            # True: `run` calls this package's operators


def listed():
    return [
        # activations of the text stream's feed-forward block: 333 tokens (an odd number)
        dict(name="quantize_text", kind="quantize", B=1, n=333, K=9728),
        # those of the image stream, 1024 x 1024, guidance pair
        dict(name="quantize_ff_image", kind="quantize", B=2, n=4096, K=6144),
        # norm before the attention, a rollout group of eight samples at 1024 x 1024
        dict(name="norm_group", kind="norm", B=8, n=4096, C=1536, affine=True, images=""),
        # requests of four sizes packed into one sequence, each with a conditioning of its own, 31 rows of padding behind them
        dict(name="norm_packed", kind="norm", B=1, n=6431, C=2432, affine=True, images="4096,1024,1024,256"),
        # the conditioning of a layer, a guidance pair: latency, and 14 MB of weights
        dict(name="linear_modulation", kind="linear", B=2, n=1, K=1536, N=9216, act="none", gate=False, residual=False, bias=True, images=""),
        # first half of the text stream's feed-forward block, guidance pair
        dict(name="linear_ff_in_text", kind="linear", B=2, n=333, K=2432, N=9728, act="gelu_tanh", gate=False, residual=False, bias=True, images=""),
        # queries, keys and values of the image stream, 1024 x 1024, guidance pair
        dict(name="linear_qkv_image", kind="linear", B=2, n=4096, K=1536, N=4608, act="none", gate=False, residual=False, bias=True, images=""),
        # second half of the feed-forward block, packed requests, each with a gate of its own, onto the residual stream
        dict(name="linear_ff_out_packed", kind="linear", B=1, n=8192, K=9728, N=2432, act="none", gate=True, residual=True, bias=True,
             images="4096,2304,1024,576,144"),
        # two small documents: latency
        dict(name="packed_tiny", kind="packed", B=1, H=2, D=64, images="144,64", texts="20,28", pad=0, mode="all", cap=0.0),
        # requests of four sizes with their prompts in one joint sequence, padded to a fixed length
        dict(name="packed_mixed", kind="packed", B=1, H=24, D=128, images="4096,1024,1024,256", texts="512,77,333,120", pad=94, mode="all", cap=0.0),
        # text that does not see its image (its states are those of every step), scores capped, a guidance pair
        dict(name="packed_text_first", kind="packed", B=2, H=24, D=64, images="2304,1024,576", texts="154,333,77", pad=0, mode="text_first", cap=30.0),
        # one sequence that is written token by token behind a prefix, capped: the largest, half of its pairs visible
        dict(name="packed_prefix", kind="packed", B=1, H=24, D=128, images="8200", texts="", pad=0, mode="prefix", cap=50.0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cut(rng, n):
    """Up to eight lengths that add up to n or less"""
    got = []
    for _ in range(rng.randint(1, 8)):
        left = n - sum(got)
        if left > 0:
            got.append(_log_uniform(rng, 1, left))
    return ",".join(map(str, got))


def _draw(rng):
    kind = rng.choice(["quantize", "norm", "linear", "linear", "linear", "packed", "packed", "packed"])
    B = _log_uniform(rng, 1, 8)
    n = 1 if rng.random() < 0.1 else _log_uniform(rng, 1, 16384)
    if kind == "quantize":
        return dict(kind=kind, B=B, n=n, K=8 * _log_uniform(rng, 2, 1216))
    if kind == "norm":
        images = _cut(rng, n) if rng.random() < 0.4 else ""
        return dict(kind=kind, B=B, n=n, C=8 * _log_uniform(rng, 8, 1216), affine=images != "" or rng.random() < 0.9, images=images)
    if kind == "linear":
        images = _cut(rng, n) if rng.random() < 0.4 else ""
        return dict(kind=kind, B=B, n=n, K=16 * _log_uniform(rng, 4, 608), N=_log_uniform(rng, 16, 9728),
                    act=rng.choice(["none", "silu", "gelu_tanh"]), gate=images != "" or rng.random() < 0.4, residual=rng.random() < 0.5,
                    bias=rng.random() < 0.8, images=images)
    mode = rng.choice(["all", "all", "text_first", "prefix"])
    images = [_log_uniform(rng, 1, 8192) for _ in range(rng.randint(1, 6))]
    texts = [] if mode == "prefix" else [rng.randint(1, 512) for _ in images]
    return dict(kind=kind, B=rng.choice([1, 1, 2]), H=rng.choice([1, 2, 5, 8, 16, 24, 24, 38]), D=rng.choice([64, 128]),
                images=",".join(map(str, images)), texts=",".join(map(str, texts)), pad=rng.choice([0, 0, rng.randint(1, 200)]),
                mode=mode, cap=rng.choice([0.0, 0.0, 15.0, 30.0, 50.0]))


def draw(rng):
    """A case of the same ranges: 1 to 16384 rows a sample, widths of 16 to 9728 in and 16 to 9728 (odd ones among them) out; 1 to 6
    documents of up to 8192 and 512 tokens, both head sizes; no more work than the listed one of its kind that has most."""
    most = {}
    for case in listed():
        w = work(case)
        b, f = most.get(case["kind"], (0.0, 0.0))
        most[case["kind"]] = (max(b, w["bytes"]), max(f, w["flops"]))
    while True:
        case = _draw(rng)
        w = work(case)
        b, f = most[case["kind"]]
        # (what the plain form of the attention makes of N x N scores grows with all pairs)
        if w["bytes"] <= max(b, 5.0e8) and w["flops"] <= f and (case["kind"] != "packed" or case["B"] * case["H"] * _tokens(case) ** 2 <= 24 * 8200 ** 2):
            return case


# ------------------------------------------------------------------------------- inputs
def _lengths(text):
    return [int(n) for n in text.split(",")] if text else []


def _tokens(case):
    return sum(_lengths(case["images"])) + sum(_lengths(case["texts"])) + case["pad"]


def _documents(lengths, n):
    """int32 [n]: the number of every row's document, -1 behind the last one"""
    d = torch.repeat_interleave(torch.arange(len(lengths)), torch.tensor(lengths, dtype=torch.long))
    return torch.cat([d, torch.full((n - d.numel(),), -1)]).int().cuda()


def _turned(lengths, b):
    b = b % max(len(lengths), 1)
    return lengths[b:] + lengths[:b]


def _normal(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


def _codes(x):
    """Rows as 8-bit integers and their scales, as a quantisation leaves them"""
    most = x.abs().amax(-1, keepdim=True)
    return torch.round(x * (127.0 / most)).to(torch.int8), (most / 127.0).squeeze(-1).contiguous()


def _inputs(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    s = dict(case)
    if case["kind"] == "quantize":
        x = torch.randn((case["B"], case["n"], case["K"]), generator=g, device="cuda")
        s["x"] = (x * torch.sigmoid(1.702 * x)).to(torch.bfloat16)             # what an activation leaves
        s["q"] = torch.zeros(x.shape, device="cuda", dtype=torch.int8)
        s["q_scale"] = torch.zeros(x.shape[:2], device="cuda")
        return s
    if case["kind"] == "packed":
        B, H, D = case["B"], case["H"], case["D"]
        images, texts = _lengths(case["images"]), _lengths(case["texts"])
        n, m = sum(images), sum(texts) + case["pad"]
        spread = 1.0 if case["cap"] == 0.0 else 3.0                             # scores that meet their cap
        s["segments"] = []
        for t in (n, m):
            if t > 0:
                # as a fused projection holds them, and the output as the next one takes it
                q, k, v = _normal(g, B, t, 3, H, D, scale=1.0).permute(2, 0, 3, 1, 4)
                q *= spread
                s["segments"].append((q, k, v, torch.empty((B, t, H, D), device="cuda", dtype=torch.bfloat16).transpose(1, 2)))
        # every sample has the documents' lengths in another order
        s["document"] = torch.stack([torch.cat([_documents(_turned(images, b), n), _documents(_turned(texts, b), m)]) for b in range(B)])
        s["order"] = None
        if case["mode"] == "text_first":
            s["order"] = (torch.arange(n + m, device="cuda") < n).int().expand(B, -1).contiguous()
        if case["mode"] == "prefix":                                            # a quarter of each document is its prefix
            at = [torch.cat([(torch.arange(L) - L // 4 + 1).clamp(min=0) for L in _turned(images, b)] + [torch.zeros(m, dtype=torch.long)]) for b in range(B)]
            s["order"] = torch.stack(at).int().cuda()
        return s
    B, n = case["B"], case["n"]
    lengths = _lengths(case["images"])
    s["document"] = torch.stack([_documents(_turned(lengths, b), n) for b in range(B)]) if lengths else None
    vectors = len(lengths) if lengths else B
    if case["kind"] == "norm":
        C = case["C"]
        s["x"] = _normal(g, B, n, C, scale=3.0) + _normal(g, 1, 1, C)           # channels of different mean, as hidden states have
        six = _normal(g, vectors, 6, C, scale=0.3)
        s["shift"], s["scale"] = (six[:, 0], six[:, 1]) if case["affine"] else (None, None)
        s["q"] = torch.zeros((B, n, C), device="cuda", dtype=torch.int8)
        s["q_scale"] = torch.zeros((B, n), device="cuda")
        return s
    K, N = case["K"], case["N"]
    x = torch.randn((B, n, K), generator=g, device="cuda")
    s["x"], s["x_scale"] = _codes(x * torch.sigmoid(1.702 * x) if case["gate"] else x)
    s["w"], s["w_scale"] = _codes(torch.randn((N, K), generator=g, device="cuda") * K ** -0.5)
    s["b"] = _normal(g, N, scale=0.1) if case["bias"] else None
    s["g"] = _normal(g, vectors, 6, N, scale=0.5)[:, 5] if case["gate"] else None
    s["r"] = _normal(g, B, n, N) if case["residual"] else None
    s["out"] = torch.zeros((B, n, N), device="cuda", dtype=torch.bfloat16)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and case["kind"] in ("linear", "packed"):
        import paper_2509_22323_amd as ra
        need = (ra.rapid_linear_int8_workspace_bytes(case["B"] * case["n"], case["N"], case["K"]) if case["kind"] == "linear"
                else ra.rapid_attn_packed_workspace_bytes(case["B"], case["H"], _tokens(case), case["D"]))
        s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------- one pass
def _own(s):
    import paper_2509_22323_amd as ra
    if s["kind"] == "quantize":
        q, q_scale = ra.rapid_quantize_rows(s["x"], s["q"], s["q_scale"])
        return q * q_scale[..., None]
    if s["kind"] == "norm":
        q, q_scale = ra.rapid_norm_modulate_int8(s["x"], s["q"], s["q_scale"], s["scale"], s["shift"], document=s["document"])
        return q * q_scale[..., None]
    if s["kind"] == "linear":
        return ra.rapid_linear_int8(s["x"], s["x_scale"], s["w"], s["w_scale"], s["out"], s["b"], s["act"], s["g"], s["r"],
                                    document=s["document"], workspace=s["workspace"])
    return ra.rapid_attn_packed(s["segments"], s["document"], s["order"], cap=s["cap"], workspace=s["workspace"])


def _quantized(y):
    """Rows y in 64 bits as whole multiples of a 127th of their largest magnitude, which is rounded to 32 bits"""
    most = y.abs().amax(-1, keepdim=True)
    codes = torch.round(127.0 * y / torch.where(most > 0, most, torch.ones_like(most)))
    return codes.float() * (most / 127.0).float()


def run(s):
    if own:
        return _own(s)
    if s["kind"] == "quantize":
        return _quantized(s["x"].double())
    if s["kind"] == "norm":
        x = s["x"].double()
        x = x - x.mean(-1, keepdim=True)
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        if s["document"] is not None:
            at = s["document"].clamp(min=0).long()
            y = y * (1.0 + s["scale"].double()[at]) + s["shift"].double()[at]
            y = torch.where((s["document"] >= 0)[..., None], y, torch.zeros_like(y))
        elif s["scale"] is not None:
            y = y * (1.0 + s["scale"].double()[:, None]) + s["shift"].double()[:, None]
        return _quantized(y)
    if s["kind"] == "linear":
        B, n, K = s["x"].shape
        y = (s["x"].float().reshape(B * n, K) @ s["w"].float().t()).reshape(B, n, -1)
        y = y * s["x_scale"][..., None] * s["w_scale"]
        if s["b"] is not None:
            y = y + s["b"].float()
        if s["act"] == "silu":
            y = y / (1.0 + torch.exp(-y))
        if s["act"] == "gelu_tanh":
            y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
        if s["g"] is not None:
            y = y * (s["g"].float()[:, None] if s["document"] is None else s["g"].float()[s["document"].clamp(min=0).long()])
        if s["r"] is not None:
            y = y + s["r"].float()
        if s["document"] is not None:
            y = torch.where((s["document"] >= 0)[..., None], y, torch.zeros_like(y))
        return y.to(torch.bfloat16)
    q, k, v = (torch.cat([t[i] for t in s["segments"]], 2).float() for i in range(3))
    z = (q @ k.transpose(-1, -2).contiguous()) * s["D"] ** -0.5
    if s["cap"] > 0.0:
        z = s["cap"] * torch.tanh(z / s["cap"])
    d = s["document"]
    hidden = (d[:, :, None] != d[:, None, :]) | (d < 0)[:, None, :]
    if s["order"] is not None:
        hidden = hidden | (s["order"][:, None, :] > s["order"][:, :, None])
    z = z.masked_fill(hidden[:, None], -math.inf)
    z = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-1e30))               # (a row of no document has no key)
    o = (z @ v) / z.sum(-1, keepdim=True).clamp(min=1e-30)
    return list(o.to(torch.bfloat16).split([t[0].shape[2] for t in s["segments"]], 2))


# ------------------------------------------------------------------------------- bounds and exact values
def work(case):
    if case["kind"] in ("quantize", "norm"):
        rows, width = case["B"] * case["n"], case["K"] if case["kind"] == "quantize" else case["C"]
        vectors = 0.0
        if case["kind"] == "norm" and case["affine"]:
            vectors = 4.0 * width * (len(_lengths(case["images"])) or case["B"])
        return {"bytes": 6.0 * rows * width + vectors, "flops": (4.0 if case["kind"] == "quantize" else 12.0) * rows * width}
    if case["kind"] == "linear":
        M, K, N = case["B"] * case["n"], case["K"], case["N"]
        vectors = (len(_lengths(case["images"])) or case["B"]) * N if case["gate"] else 0
        return {"bytes": 1.0 * M * K + N * K + 4.0 * (M + N) + 2.0 * (M * N * (2 if case["residual"] else 1) + (N if case["bias"] else 0) + vectors),
                "flops": 2.0 * M * K * N}
    images, texts = _lengths(case["images"]), _lengths(case["texts"])
    pairs = 0
    for i, n in enumerate(images):
        m = texts[i] if texts else 0
        if case["mode"] == "all":
            pairs += (n + m) ** 2
        elif case["mode"] == "text_first":
            pairs += n * (n + m) + m * m
        else:
            p, q = n // 4, n - n // 4                                           # the prefix, and tokens that see those before them
            pairs += p * p + q * p + q * (q + 1) // 2
    return {"bytes": 8.0 * case["B"] * case["H"] * _tokens(case) * case["D"] + 4.0 * case["B"] * _tokens(case),
            "flops": 4.0 * case["B"] * case["H"] * case["D"] * pairs}


def _exact_rows(y):
    """In 64 bits: the nearest whole multiple (ties to the even one) of every row's step"""
    top = y.abs().max(dim=-1, keepdim=True).values
    return torch.where(top > 0, (y * 127 / top).round() * top / 127, torch.zeros_like(y))


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "quantize":
        return _exact_rows(s["x"].double())
    if case["kind"] in ("norm", "linear"):
        vector = {}
        for name in ("scale", "shift", "g"):
            t = s.get(name)
            if t is not None:
                t = t.double()
                if s["document"] is None:
                    vector[name] = t.unsqueeze(1)
                else:
                    vector[name] = torch.nn.functional.embedding(s["document"].relu().long(), t.contiguous())
        if case["kind"] == "norm":
            variance, mean = torch.var_mean(s["x"].double(), dim=-1, correction=0, keepdim=True)
            y = (s["x"].double() - mean) / (variance + 1e-6).sqrt()
            if vector:
                y = torch.addcmul(vector["shift"], y, 1 + vector["scale"])
        else:
            B, n, K = s["x"].shape
            y = torch.mm(s["x"].double().view(B * n, K) * s["x_scale"].double().view(-1, 1), (s["w"].double() * s["w_scale"].double()[:, None]).t().contiguous())
            y = y.view(B, n, case["N"])
            if case["bias"]:
                y.add_(s["b"].double())
            if case["act"] == "silu":
                y.mul_(torch.sigmoid(y))
            elif case["act"] == "gelu_tanh":
                y.mul_(torch.sigmoid(math.sqrt(8.0 / math.pi) * (y + 0.044715 * y.pow(3))))
            if case["gate"]:
                y.mul_(vector["g"])
            if case["residual"]:
                y.add_(s["r"].double())
        if s["document"] is not None:
            y[s["document"] < 0] = 0.0
        return _exact_rows(y) if case["kind"] == "norm" else y
    made = [torch.zeros(t[0].shape, dtype=torch.float64, device="cuda") for t in s["segments"]]
    first = s["segments"][0][0].shape[2]
    for b in range(case["B"]):
        d = s["document"][b]
        for number in range(len(_lengths(case["images"]))):                     # the documents one by one, each in an order of its tokens
            at = (d == number).nonzero().squeeze(1)
            for h in range(case["H"]):
                q, k, v = (torch.cat([t[i][b, h] for t in s["segments"]])[at].double() for i in range(3))
                z = torch.mm(q, k.t().contiguous()) / math.sqrt(case["D"])
                if case["cap"] > 0.0:
                    z = case["cap"] * torch.tanh(z / case["cap"])
                if s["order"] is not None:
                    o = s["order"][b, at]
                    z[o[:, None] < o[None, :]] = -math.inf
                y = torch.mm(torch.softmax(z, -1), v)
                made[0][b, h, at[at < first]] = y[at < first]
                if len(made) > 1:
                    made[1][b, h, at[at >= first] - first] = y[at >= first]
    return made
