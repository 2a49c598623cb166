"""Host-only checks of layers in 8 bits over packed sequences: exported symbols, every refusal of the C entries before any launch, and the
refusals of the Python forms."""
import ctypes
import os
import re

import pytest
import torch

import paper_2509_22323_amd as ra
from paper_2509_22323_amd import binding
from paper_2509_22323_amd.binding import Rows, Segment

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "rapid_packed.h")).read()
A = 0x10000          # fake aligned "device" addresses: never dereferenced, every call below fails its checks
S = ra.STATUS
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE, ALIAS = (S["RAPID_ERR_" + n] for n in (
    "NULL", "SHAPE", "UNSUPPORTED", "ALIGN", "WORKSPACE", "ALIAS"))


def test_header_and_library_agree():
    declared = re.findall(r"RAPID_API\s+[\w\s\*]+?\b(rapid_\w+)\s*\(", HEADER)
    assert set(declared) == set(binding.PACKED_EXPORTS)
    ra.library()
    lib = ctypes.CDLL(ra.library_path())
    for name in declared:
        assert hasattr(lib, name), name
        assert name in ra.__all__


def quantize(x=(A, 0, 64), q=(3 * A, 0, 64), scale=5 * A, B=1, n=4, K=64):
    rows = [None if t is None else ctypes.byref(Rows(*t)) for t in (x, q)]
    return ra.library().rapid_quantize_rows(*rows, scale, B, n, K, None)


def norm(x=(A, 0, 64), q=(3 * A, 0, 64), q_scale=5 * A, scale=6 * A, ss=64, shift=7 * A, hs=64, document=None, documents=0, B=1, n=4, C=64, eps=1e-6):
    rows = [None if t is None else ctypes.byref(Rows(*t)) for t in (x, q)]
    return ra.library().rapid_norm_modulate_int8(*rows, q_scale, scale, ss, shift, hs, document, documents, B, n, C, eps, None)


ROWS = [
    (dict(x=None), NULL), (dict(q=None), NULL), (dict(x=(None, 0, 64)), NULL), (dict(q=(None, 0, 64)), NULL),
    (dict(B=0), SHAPE), (dict(n=0), SHAPE), (dict(n=-1), SHAPE), (dict(n=(1 << 22) + 1), SHAPE), (dict(B=1 << 12, n=(1 << 10) + 1), SHAPE),
    (dict(x=(A, 0, -64)), SHAPE), (dict(x=(A, 0, (1 << 22) + 8)), SHAPE), (dict(q=(3 * A, 0, 56)), SHAPE),
    (dict(B=2, x=(A, 256, 64), q=(3 * A, 248, 64)), SHAPE), (dict(B=2, x=(A, -8, 64), q=(3 * A, 256, 64)), SHAPE),
    (dict(B=2, x=(A, (1 << 40) + 8, 64), q=(3 * A, 256, 64)), SHAPE),
    (dict(x=(A + 8, 0, 64)), ALIGN), (dict(q=(3 * A + 4, 0, 64)), ALIGN), (dict(x=(A, 0, 68)), ALIGN), (dict(q=(3 * A, 0, 68)), ALIGN),
    (dict(q=(A, 0, 64)), ALIAS),
]


@pytest.mark.parametrize("kw,code", ROWS + [
    (dict(scale=None), NULL), (dict(K=0), SHAPE), (dict(K=60), UNSUPPORTED), (dict(K=(1 << 17) + 8), UNSUPPORTED), (dict(scale=5 * A + 2), ALIGN),
    (dict(scale=A), ALIAS), (dict(scale=3 * A), ALIAS)], ids=str)
def test_quantize_refusals(kw, code):
    assert quantize(**kw) == code


@pytest.mark.parametrize("kw,code", ROWS + [
    (dict(q_scale=None), NULL), (dict(scale=None), NULL), (dict(shift=None), NULL), (dict(C=0), SHAPE), (dict(eps=-1.0), SHAPE),
    (dict(eps=float("nan")), SHAPE), (dict(document=8 * A), SHAPE), (dict(document=8 * A, documents=-1), SHAPE),
    (dict(B=2, x=(A, 256, 64), q=(3 * A, 256, 64), ss=-64), SHAPE), (dict(document=8 * A, documents=2, hs=-8), SHAPE),
    (dict(C=60), UNSUPPORTED), (dict(C=16392, x=(A, 0, 16392), q=(3 * A, 0, 16392)), UNSUPPORTED),
    (dict(q_scale=5 * A + 2), ALIGN), (dict(scale=6 * A + 8), ALIGN), (dict(shift=7 * A + 2), ALIGN), (dict(document=8 * A + 2, documents=3), ALIGN),
    (dict(document=8 * A, documents=2, ss=68), ALIGN),
    (dict(q_scale=A), ALIAS), (dict(q_scale=6 * A), ALIAS), (dict(q=(7 * A, 0, 64)), ALIAS), (dict(document=3 * A, documents=1), ALIAS)], ids=str)
def test_norm_refusals(kw, code):
    assert norm(**kw) == code


def linear(x=(A, 0, 64), xs=11 * A, w=2 * A, ws=64, wsc=12 * A, bias=None, y=(3 * A, 0, 32), act=0, gate=None, gs=0, res=None, document=None,
           documents=0, B=1, n=4, N=32, K=64, work=None, work_bytes=0):
    rows = [None if t is None else ctypes.byref(Rows(*t)) for t in (x, y, res)]
    return ra.library().rapid_linear_int8(rows[0], xs, w, ws, wsc, bias, rows[1], act, gate, gs, rows[2], document, documents, B, n, N, K, work,
                                          work_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(w=None), NULL), (dict(xs=None), NULL), (dict(wsc=None), NULL), (dict(x=(None, 0, 64)), NULL),
    (dict(y=(None, 0, 32)), NULL), (dict(res=(None, 0, 32)), NULL),
    (dict(B=0), SHAPE), (dict(n=0), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(B=-1), SHAPE), (dict(n=-5), SHAPE),
    (dict(N=(1 << 22) + 1), SHAPE), (dict(K=(1 << 22) + 16), SHAPE), (dict(B=1 << 16, n=1 << 15), SHAPE), (dict(n=(1 << 31) - 100), SHAPE),
    (dict(x=(A, 0, -16)), SHAPE), (dict(x=(A, 0, (1 << 22) + 16)), SHAPE), (dict(x=(A, -16, 64), B=2, y=(3 * A, 128, 32)), SHAPE),
    (dict(ws=48), SHAPE), (dict(ws=(1 << 22) + 16), SHAPE), (dict(gate=A, gs=-1, B=2, x=(A, 256, 64), y=(3 * A, 128, 32)), SHAPE),
    (dict(y=(3 * A, 0, 31)), SHAPE), (dict(B=2, x=(A, 256, 64), y=(3 * A, 127, 32)), SHAPE), (dict(B=2, x=(A, 1 << 30, 64), y=(3 * A, 128, 32)), SHAPE),
    (dict(document=13 * A), SHAPE), (dict(document=13 * A, documents=2, gate=14 * A, gs=-32), SHAPE),
    (dict(K=72, x=(A, 0, 80), ws=80), UNSUPPORTED), (dict(K=1 << 17, x=(A, 0, 1 << 17), ws=1 << 17), UNSUPPORTED), (dict(act=3), UNSUPPORTED),
    (dict(act=-1), UNSUPPORTED),
    (dict(x=(A + 8, 0, 64)), ALIGN), (dict(w=2 * A + 8), ALIGN), (dict(x=(A, 0, 72)), ALIGN), (dict(ws=72), ALIGN), (dict(xs=11 * A + 2), ALIGN),
    (dict(wsc=12 * A + 1), ALIGN), (dict(document=13 * A + 2, documents=1), ALIGN), (dict(B=2, x=(A, 264, 64), y=(3 * A, 128, 32)), ALIGN),
    (dict(y=(3 * A + 1, 0, 32)), ALIGN), (dict(bias=A + 1), ALIGN), (dict(gate=A + 1), ALIGN), (dict(res=(A + 1, 0, 32)), ALIGN),
    (dict(y=(A, 0, 32)), ALIAS), (dict(y=(2 * A, 0, 32)), ALIAS), (dict(y=(11 * A, 0, 32)), ALIAS), (dict(y=(12 * A, 0, 32)), ALIAS),
    (dict(bias=3 * A), ALIAS), (dict(gate=3 * A), ALIAS), (dict(document=3 * A, documents=1), ALIAS), (dict(res=(3 * A, 0, 40)), ALIAS),
    (dict(B=2, x=(A, 256, 64), y=(3 * A, 128, 32), res=(3 * A, 256, 32)), ALIAS),
    (dict(work=A + 8, work_bytes=1 << 30), WORKSPACE),
], ids=str)
def test_linear_refusals(kw, code):
    assert linear(**kw) == code


SEG = dict(q=A, k=2 * A, v=3 * A, o=4 * A, n=4, in_b=512, in_h=256, in_n=64, out_b=512, out_h=256, out_n=64)
OTHER = dict(q=5 * A, k=6 * A, v=7 * A, o=8 * A)


def attend(segs=({},), B=1, H=2, D=64, document=9 * A, ds=4, order=None, os=4, cap=0.0, scale=0.0, work=10 * A, work_bytes=1 << 40, n_segments=None):
    arr = (Segment * max(len(segs), 1))(*(Segment(*{**SEG, **s}.values()) for s in segs)) if segs is not None else None
    n = len(segs or ()) if n_segments is None else n_segments
    return ra.library().rapid_attn_packed(arr, n, B, H, D, document, ds, order, os, cap, scale, work, work_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(segs=None, n_segments=1), NULL), (dict(segs=()), NULL), (dict(document=None), NULL), (dict(work=None), NULL),
    *((dict(segs=({name: None},)), NULL) for name in "qkvo"), *((dict(segs=({}, {**OTHER, name: None})), NULL) for name in "qkvo"),
    (dict(segs=({},) * 3), SHAPE), (dict(B=0), SHAPE), (dict(H=-1), SHAPE), (dict(B=1 << 10, H=1 << 10), SHAPE), (dict(segs=({"n": 0},)), SHAPE),
    (dict(segs=({"n": (1 << 22) + 1},)), SHAPE), (dict(segs=({"n": 1 << 22}, OTHER)), SHAPE), (dict(segs=({"in_n": 56},)), SHAPE),
    (dict(segs=({"out_n": 0},)), SHAPE), (dict(segs=({"in_n": (1 << 23) + 8},)), SHAPE), (dict(segs=({"in_n": 1 << 23},)), SHAPE), (dict(segs=({"out_n": 1 << 23},)), SHAPE),
    (dict(B=1 << 8, H=1 << 8, segs=({"n": 1 << 15},)), SHAPE), (dict(segs=({"in_h": -64},)), SHAPE),
    (dict(segs=({"out_h": (1 << 40) + 8},)), SHAPE), (dict(B=2, segs=({"in_b": -8},)), SHAPE), (dict(B=2, ds=-1), SHAPE),
    (dict(B=2, order=A, os=-4), SHAPE), (dict(B=2, ds=(1 << 40) + 1), SHAPE), (dict(B=1 << 9, H=1 << 9, segs=({"n": 1 << 18},)), SHAPE),
    (dict(D=96), UNSUPPORTED), (dict(cap=-1.0), UNSUPPORTED), (dict(cap=float("inf")), UNSUPPORTED), (dict(cap=float("nan")), UNSUPPORTED),
    (dict(scale=float("nan")), UNSUPPORTED), (dict(scale=float("inf")), UNSUPPORTED),
    *((dict(segs=({name: 20 * A + 8},)), ALIGN) for name in "qkvo"), (dict(segs=({"in_n": 68},)), ALIGN), (dict(segs=({"out_h": 260},)), ALIGN),
    (dict(document=9 * A + 2), ALIGN), (dict(order=9 * A + 2), ALIGN), (dict(work=10 * A + 8), ALIGN),
    (dict(work_bytes=0), WORKSPACE),
    *((dict(segs=({"o": at * A},)), ALIAS) for at in (1, 2, 3)), *((dict(segs=({}, {**OTHER, "o": at * A})), ALIAS) for at in (1, 2, 3, 4, 5, 6, 7)),
    (dict(segs=({"o": 7 * A}, OTHER)), ALIAS),
], ids=str)
def test_attention_refusals(kw, code):
    assert attend(**kw) == code


def test_strides_of_dimensions_of_size_one_are_not_looked_at():
    odd = dict(in_b=-3, in_h=-3, in_n=-3, out_b=1, out_h=1, out_n=1, n=1)
    assert attend(segs=(odd,), B=1, H=1, ds=-7, order=A, os=-7, work_bytes=0) == WORKSPACE


@pytest.mark.parametrize("size", [(0, 1, 64, 64), (1, 0, 64, 64), (1, 1, 0, 64), (1, 1, (1 << 22) + 1, 64), (1, 1, 64, 96), (1 << 10, 1 << 10, 64, 64),
                                  (1 << 32, 1, 64, 64), (1, 1, 1 << 32, 64), (1 << 8, 1 << 8, 1 << 15, 64)], ids=str)
def test_workspaces_of_sizes_that_are_refused(size):
    assert ra.rapid_attn_packed_workspace_bytes(*size) == 0


@pytest.mark.parametrize("size", [(0, 64, 64), (64, 0, 64), (64, 64, 0), (64, 64, 72), (64, 64, 1 << 17), (300 + (1 << 32), 320, 4096), (300, 320, 4096 + (1 << 32)),
                                  (300, (1 << 22) + 1, 4096), ((1 << 31) - 200, 64, 64)], ids=str)
def test_workspaces_of_products_that_are_refused(size):
    assert ra.rapid_linear_int8_workspace_bytes(*size) == 0


def test_python_forms_take_tensors_of_the_gpu_alone():
    x, q8, s = torch.zeros((1, 4, 64), dtype=torch.bfloat16), torch.zeros((1, 4, 64), dtype=torch.int8), torch.zeros((1, 4))
    q = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16)
    for call in (lambda: ra.rapid_quantize_rows(x, q8, s), lambda: ra.rapid_norm_modulate_int8(x, q8, s), lambda: ra.rapid_quantize_rows(None, q8, s),
                 lambda: ra.rapid_linear_int8(q8, s, q8[0], s[0], x), lambda: ra.rapid_attn_packed([(q, q, q, q)], torch.zeros(4, dtype=torch.int32))):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        ra.rapid_attn_packed([], torch.zeros(4, dtype=torch.int32))


@pytest.mark.skipif(binding._load_native().__class__ is binding._NoNative, reason="the native calls are not built for this torch")
def test_native_forms_leave_other_tensors_to_the_python_form():
    x, q8, s = torch.zeros((1, 4, 64), dtype=torch.bfloat16), torch.zeros((1, 4, 64), dtype=torch.int8), torch.zeros((1, 4))
    q, d = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    native = binding._load_native()
    assert native.quantize(x, q8, s) is None and native.quantize(x) is None
    assert native.modulate8(x, q8, s, None, None, 1e-6, None) is None
    assert native.linear8(q8, s, q8[0], s[0], x, None, "none", None, None, None, None) is None
    assert native.packed_attention([(q, q, q, q)], d, None, 0.0, 0.0, s) is None
