"""rapid_linear against the fp64 oracle."""
import numpy as np
import pytest
import torch

import paper_2509_22323_amd as ra
from layer_common import BF16_STEP, NAN, assert_within, inside, normal, untouched_around, widen
from oracle import layer_oracle as lo

pytestmark = pytest.mark.gpu


def bound(x, w, bias, act, gate, residual, want):
    """What rounding can do to an output.  Products of two bf16 are exact in fp32; each of the K additions rounds by at most one
    step of the sum's absolute values (2^-23, whichever way the matrix unit rounds): e0.  Activations grow an error by 1.13 at
    most (their largest slopes are 1.10 and 1.13) and round a handful of times themselves: z by 2^-20 relative covers exp2's and
    the reciprocal's last place and their argument's (|t| sigma(1 - sigma) < 0.28).  Gate and residual: one rounding each.
    Then half a step of bf16, and half of its smallest number."""
    K = x.shape[-1]
    z = np.matmul(x, w.T) + (0 if bias is None else bias)
    e = (K + 1) * 2.0 ** -23 * (np.matmul(np.abs(x), np.abs(w).T) + (0 if bias is None else np.abs(bias)))
    if act != "none":
        e = 1.13 * e + 2.0 ** -20 * np.abs(z)
    a = np.abs(lo.activation(z, act))
    if gate is not None:
        e = np.abs(gate)[:, None] * (e + 2.0 ** -24 * a)
        a = np.abs(gate)[:, None] * a
    if residual is not None:
        e = e + 2.0 ** -24 * (a + np.abs(residual) + e)
    return e + BF16_STEP * (np.abs(want) + e) + 2.0 ** -134


def check(B, n, K, N, act="none", bias=True, gate=False, residual=False, seed=1, workspace=True, in_place=False, pads=(2, 3, 8)):
    """Every tensor lies inside a buffer of NaN (rows before and behind, columns behind): nothing of it may reach a result,
    nothing around the result may change."""
    xt, wt = normal((B, n, K), seed), normal((N, K), seed + 1, K ** -0.5)
    before, after, columns = pads
    x, _ = inside(xt, before, after, columns)
    w = inside(wt[None], 1, 2, columns)[0][0]
    b = normal((N,), seed + 2, 0.3) if bias else None
    g = normal((B, 3, N), seed + 3)[:, 1] if gate else None
    r = normal((B, n, N), seed + 4) if residual else None
    want = lo.linear(*(None if t is None else widen(t) for t in (xt, wt, b)), act, *(None if t is None else widen(t) for t in (g, r)))
    e = bound(*(None if t is None else widen(t) for t in (xt, wt, b)), act, *(None if t is None else widen(t) for t in (g, r)), want)
    outs = []
    need = ra.rapid_linear_workspace_bytes(B * n, N, K)
    for ws in (None, torch.full((need,), 0xAB, dtype=torch.uint8, device="cuda")) if workspace else (None,):
        out, big = inside(torch.full((B, n, N), NAN, dtype=torch.bfloat16, device="cuda"), before, after, columns)
        res = r
        if in_place and residual:
            out.copy_(r)
            res = out
        got = ra.rapid_linear(x, w, out, b, act, g, res, ws)
        assert got is out
        assert_within(out, want, e, f"{(B, n, K, N, act)}")
        assert untouched_around(out, big)
        outs.append(out.clone())
    return outs


SIZES = [(1, 1, 8, 1), (1, 1, 64, 16), (2, 1, 256, 1536), (1, 3, 72, 5), (8, 1, 1536, 333), (1, 16, 328, 129), (1, 17, 1000, 64),
         (3, 33, 200, 66), (1, 64, 512, 512), (2, 77, 640, 384), (1, 100, 2432, 100), (1, 129, 136, 257), (2, 333, 96, 260),
         (1, 255, 1544, 1024), (1, 257, 64, 511), (5, 1, 9728, 48), (1, 40, 4864, 320), (7, 130, 104, 1000), (1, 1030, 520, 770),
         (1, 2048, 256, 2048), (40, 7, 192, 192), (300, 1, 136, 72)]


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_sizes(size):
    B, n, K, N = size
    check(B, n, K, N, seed=sum(size))


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 7, 8, 9])
@pytest.mark.parametrize("K,N", [(8, 3), (512, 64), (1544, 131), (2560, 33), (6144, 1536)])
def test_a_handful_of_rows(rows, K, N):
    check(rows, 1, K, N, "silu", True, True, rows % 2 == 0, seed=rows)
    check(1, rows, K, N, seed=rows)


@pytest.mark.parametrize("act", ["none", "silu", "gelu_tanh"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("gate,residual", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("size", [(2, 1, 264, 100), (2, 45, 136, 67), (3, 200, 264, 324)], ids=str)
def test_epilogues(size, act, bias, gate, residual):
    check(*size, act, bias, gate, residual, seed=7, workspace=False)


@pytest.mark.parametrize("size", [(2, 1, 136, 64), (2, 50, 136, 64), (2, 300, 512, 640)], ids=str)
def test_residual_in_place(size):
    check(*size, "none", True, True, True, in_place=True)


@pytest.mark.parametrize("size", [(1, 5, 64, 63), (1, 5, 64, 64), (1, 150, 64, 130)], ids=str)
def test_unaligned_outputs(size):
    """Output rows that start at odd elements."""
    B, n, K, N = size
    x, w = normal((n, K), 3), normal((N, K), 4, K ** -0.5)
    flat = torch.full((n * (N + 3) + 1,), NAN, dtype=torch.bfloat16, device="cuda")
    out = flat[1:].view(n, N + 3)[:, :N]
    ra.rapid_linear(x, w, out)
    want = lo.linear(widen(x)[None], widen(w))[0]
    assert_within(out, want, bound(widen(x)[None], widen(w), None, "none", None, None, want[None])[0])
    assert torch.isnan(flat[1:].view(n, N + 3)[:, N:]).all() and torch.isnan(flat[0])


def test_samples_of_a_joint_buffer_and_samples_inside_tokens():
    B, n, K, N = 3, 70, 64, 96
    x, w = normal((n, B, K), 5).transpose(0, 1), normal((N, K), 6, K ** -0.5)      # [B, n, K], the samples of a token side by side
    out = torch.full((n, B, N), NAN, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    one = normal((1, n, K), 8).expand(B, n, K)                                     # the same rows for every sample
    for t in (x, one):
        ra.rapid_linear(t, w, out)
        want = lo.linear(widen(t), widen(w))
        assert_within(out, want, bound(widen(t), widen(w), None, "none", None, None, want))


def test_far_activations():
    """exp over- and underflows on the way; the limits are 0 and z."""
    z = torch.tensor([[0.0, 1e-30, 1.0, -1.0, 30.0, -30.0, 200.0, -200.0, 1e4, -1e4, 1e18, -1e18, 3e38, -3e38, 1e-38, -0.5]],
                     device="cuda").to(torch.bfloat16)
    w = torch.eye(16, dtype=torch.bfloat16, device="cuda")
    for act in ("silu", "gelu_tanh"):
        out = ra.rapid_linear(z, w, torch.empty_like(z), activation=act)
        with np.errstate(over="ignore"):
            want = lo.activation(widen(z), act)
        assert_within(out, want, (BF16_STEP + 2.0 ** -20) * np.abs(want) + 2.0 ** -126, act)   # (below that fp32 may flush)


def test_values_that_are_not_numbers_stay_in_their_rows_and_columns():
    n, K, N = 150, 136, 140
    x, w = normal((n, K), 11), normal((N, K), 12, K ** -0.5)
    clean = ra.rapid_linear(x, w, torch.empty((n, N), dtype=torch.bfloat16, device="cuda")).clone()
    x[7, 135], w[130, 3] = NAN, float("inf")
    got = ra.rapid_linear(x, w, torch.empty_like(clean))
    assert torch.isnan(got[7]).all() and not torch.isfinite(got[:, 130]).any()
    rows, columns = [i for i in range(n) if i != 7], [j for j in range(N) if j != 130]
    assert torch.equal(got[rows][:, columns], clean[rows][:, columns])


def test_repeated_calls_give_the_same_bits():
    for B, n, K, N in ((2, 1, 1536, 640), (1, 100, 4096, 256), (1, 700, 2048, 900)):
        first = check(B, n, K, N, "gelu_tanh", seed=21)
        again = check(B, n, K, N, "gelu_tanh", seed=21)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_whole_numbers_are_exact():
    """Small whole numbers: every sum is exact in fp32 and below 2^8, so that the result is too, whatever the order."""
    rng = np.random.default_rng(5)
    for n, K, N in ((1, 200, 100), (90, 200, 300), (600, 264, 300)):
        x = torch.from_numpy(rng.integers(-1, 2, (n, K)).astype(np.float32)).to(torch.bfloat16).cuda()
        w = torch.from_numpy(rng.integers(-1, 2, (N, K)).astype(np.float32)).to(torch.bfloat16).cuda()
        got = ra.rapid_linear(x, w, torch.empty((n, N), dtype=torch.bfloat16, device="cuda"))
        np.testing.assert_array_equal(widen(got), widen(x) @ widen(w).T)


# (one of each tile: 256 x 192, 256 x 160, 256 x 256, 128 x 128 in pieces and whole; several tiles a workgroup; ends of K and N inside)
LARGE = [(2, 4000, 1544, 4600), (1, 8191, 3000, 2431), (2, 20000, 200, 1000), (1, 1024, 6144, 1536), (3, 1000, 1000, 2500), (1, 16000, 512, 4097),
         (40, 201, 264, 2000), (9000, 1, 704, 1500)]


@pytest.mark.parametrize("size", LARGE, ids=str)
@pytest.mark.parametrize("gated", [False, True])
def test_large(size, gated):
    B, n, K, N = size
    g = torch.Generator("cuda").manual_seed(sum(size))

    def make(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16)

    x, w, b = inside(make(B, n, K), 1, 2, 8)[0], make(N, K, scale=K ** -0.5), make(N, scale=0.3)
    gate, res = (make(B, N), make(B, n, N)) if gated else (None, None)
    out, big = inside(torch.full((B, n, N), NAN, dtype=torch.bfloat16, device="cuda"), 1, 1, 3)
    ra.rapid_linear(x, w, out, b, "gelu_tanh" if gated else "none", gate, res)
    assert torch.isfinite(out).all() and untouched_around(out, big)
    m = np.unique(np.concatenate([[0, B * n - 1], np.random.default_rng(1).integers(0, B * n, 300), np.arange(max(0, B * n - 260), B * n, 37)]))
    s, r = torch.from_numpy(m // n).cuda(), torch.from_numpy(m % n).cuda()
    rows = [widen(t) for t in (x[s, r], w, b)] + ([widen(gate[s]), widen(res[s, r])] if gated else [None, None])
    act = "gelu_tanh" if gated else "none"
    args = (rows[0][:, None], rows[1], rows[2], act, rows[3], None if rows[4] is None else rows[4][:, None])
    want = lo.linear(*args)
    assert_within(out[s, r][:, None], want, bound(*args, want), str(size))


def test_samples_shorter_than_a_tile():
    """A gate of its own for every sample, many samples in one tile of rows."""
    check(40, 7, 192, 192, "silu", True, True, True, seed=31)
    check(300, 1, 136, 72, "none", True, True, True, seed=32)
    check(9, 30, 2432, 100, "gelu_tanh", False, True, True, seed=33)


def test_offsets_beyond_32_bits():
    """x and y of more than 2^32 bytes each, w of rows far apart."""
    n, K, N = 300000, 8192, 8000
    x = torch.zeros((n, K), dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 1, 131071, 262143, 262144, 299998, 299999], device="cuda")
    x[rows] = normal((7, K), 41)
    w = torch.full((N, 8200), NAN, dtype=torch.bfloat16, device="cuda")[:, :K]
    w.copy_(normal((N, K), 42, K ** -0.5))
    out = torch.full((n, N), NAN, dtype=torch.bfloat16, device="cuda")
    ra.rapid_linear(x, w, out)
    args = (widen(x[rows])[None], widen(w))
    want = lo.linear(*args)
    assert_within(out[rows][None], want, bound(*args, None, "none", None, None, want))
    out[rows] = 0
    assert not out.any()                                                           # every other row of x is zero


def test_without_a_workspace():
    for B, n, K, N in ((1, 100, 2432, 100), (1, 1024, 6144, 1536)):
        assert ra.rapid_linear_workspace_bytes(B * n, N, K) > 0
        x, w = normal((n, K), 51), normal((N, K), 52, K ** -0.5)
        out = torch.empty((n, N), dtype=torch.bfloat16, device="cuda")
        rows = ra.binding.Rows(x.data_ptr(), 0, K), ra.binding.Rows(out.data_ptr(), 0, N)
        status = ra.library().rapid_linear(rows[0], w.data_ptr(), K, None, rows[1], 0, None, 0, None, 1, n, N, K, None, 0,
                                           torch.cuda.current_stream().cuda_stream)
        assert status == 0
        args = (widen(x)[None], widen(w))
        want = lo.linear(*args)
        assert_within(out[None], want, bound(*args, None, "none", None, None, want))
        small = torch.empty(64, dtype=torch.uint8, device="cuda")
        with pytest.raises(ra.RapidAttnError) as e:
            ra.rapid_linear(x, w, out, workspace=small)
        assert e.value.status == ra.STATUS["RAPID_ERR_WORKSPACE"]


@pytest.mark.parametrize("size", [(2, 333, 2432, 9728), (1, 666, 2440, 9721), (2, 2048, 6144, 1536), (3, 683, 4000, 4090)], ids=str)
def test_middling_products(size):
    """Fewer large tiles than the card has CUs, or not many more: 256 x 128 and 256 x 160."""
    test_large(size, True)
    test_large(size, False)


@pytest.mark.parametrize("rows", [2, 90])
def test_rows_that_are_one_row(rows):
    """Inputs of stride 0: the same row of x for every token, the same residual for every sample or every token."""
    one, w, b = normal((3, 1, 200), 1), normal((130, 200), 2, 200 ** -0.5), normal((130,), 3)
    for r in (normal((1, rows, 130), 4).expand(3, -1, -1), normal((3, 1, 130), 5).expand(-1, rows, -1)):
        out = torch.full((3, rows, 130), NAN, dtype=one.dtype, device="cuda")
        ra.rapid_linear(one.expand(-1, rows, -1), w, out, b, "silu", b, r)
        args = [widen(one.expand(-1, rows, -1)), widen(w), widen(b), "silu", widen(b.expand(3, -1)), widen(r)]
        want = lo.linear(*args)
        assert_within(out, want, bound(*args, want), str(rows))
