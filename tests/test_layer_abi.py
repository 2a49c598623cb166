"""Host-only checks of the operators around the attention: exported symbols, every refusal of the C entries before any launch, and the
refusals of the Python forms."""
import ctypes
import os
import re

import pytest
import torch

import paper_2509_22323_amd as ra
from paper_2509_22323_amd import binding
from paper_2509_22323_amd.binding import QkSegment, Rows

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "rapid_layer.h")).read()
A = 0x10000          # fake aligned "device" addresses: never dereferenced, every call below fails its checks
S = ra.STATUS
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE, ALIAS = (S["RAPID_ERR_" + n] for n in (
    "NULL", "SHAPE", "UNSUPPORTED", "ALIGN", "WORKSPACE", "ALIAS"))


def test_header_and_library_agree():
    declared = re.findall(r"RAPID_API\s+[\w\s\*]+?\b(rapid_\w+)\s*\(", HEADER)
    assert set(declared) == set(binding.LAYER_EXPORTS)
    ra.library()
    lib = ctypes.CDLL(ra.library_path())
    for name in declared:
        assert hasattr(lib, name), name
    for names, prefix in ((binding.ACTIVATIONS, "RAPID_ACT_"), (binding.ROPE_SCALINGS, "RAPID_ROPE_"), (binding.ROPE_LAYOUTS, "RAPID_ROPE_")):
        for name, value in names.items():
            c = {"half": "halves", "none": "plain" if prefix == "RAPID_ROPE_" else "none"}.get(name, name).upper()
            assert re.search(rf"{prefix}{c}\s*=\s*{value}\b", HEADER), name


def linear(x=(A, 0, 64), w=2 * A, ws=64, bias=None, y=(3 * A, 0, 32), act=0, gate=None, gs=0, res=None, B=1, n=4, N=32, K=64,
           work=None, work_bytes=0):
    rows = [None if t is None else ctypes.byref(Rows(*t)) for t in (x, y, res)]
    return ra.library().rapid_linear(rows[0], w, ws, bias, rows[1], act, gate, gs, rows[2], B, n, N, K, work, work_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(w=None), NULL), (dict(x=(None, 0, 64)), NULL), (dict(y=(None, 0, 32)), NULL),
    (dict(res=(None, 0, 32)), NULL),
    (dict(B=0), SHAPE), (dict(n=0), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(B=-1), SHAPE), (dict(n=-5), SHAPE),
    (dict(N=(1 << 22) + 1), SHAPE), (dict(K=(1 << 22) + 8), SHAPE), (dict(B=1 << 16, n=1 << 15), SHAPE),
    (dict(n=(1 << 31) - 100), SHAPE),
    (dict(x=(A, 0, -8)), SHAPE), (dict(x=(A, 0, (1 << 22) + 8)), SHAPE), (dict(x=(A, -8, 64), B=2, y=(3 * A, 128, 32)), SHAPE),
    (dict(ws=56), SHAPE), (dict(ws=(1 << 22) + 8), SHAPE), (dict(gate=A, gs=-1, B=2, x=(A, 256, 64), y=(3 * A, 128, 32)), SHAPE),
    (dict(y=(3 * A, 0, 31)), SHAPE), (dict(B=2, x=(A, 256, 64), y=(3 * A, 127, 32)), SHAPE), (dict(B=2, x=(A, 256, 64), y=(3 * A, 0, 32)), SHAPE),
    (dict(B=2, x=(A, 256, 64), y=(3 * A, 32, 63)), SHAPE), (dict(B=2, n=1, x=(A, 64, 0), y=(3 * A, 31, 0)), SHAPE),
    (dict(B=2, x=(A, 1 << 30, 64), y=(3 * A, 128, 32)), SHAPE),
    (dict(K=60), UNSUPPORTED), (dict(act=3), UNSUPPORTED), (dict(act=-1), UNSUPPORTED),
    (dict(x=(A + 8, 0, 64)), ALIGN), (dict(w=2 * A + 2), ALIGN), (dict(x=(A, 0, 68)), ALIGN), (dict(ws=68), ALIGN),
    (dict(B=2, x=(A, 260, 64), y=(3 * A, 128, 32)), ALIGN), (dict(y=(3 * A + 1, 0, 32)), ALIGN), (dict(bias=A + 1), ALIGN),
    (dict(gate=A + 1), ALIGN), (dict(res=(A + 1, 0, 32)), ALIGN),
    (dict(y=(A, 0, 32)), ALIAS), (dict(y=(2 * A, 0, 32)), ALIAS),
    (dict(work=A + 8, work_bytes=1 << 30), WORKSPACE),
], ids=str)
def test_linear_refusals(kw, code):
    assert linear(**kw) == code


def modulate(x=(A, 0, 64), y=(3 * A, 0, 64), scale=4 * A, ss=64, shift=5 * A, hs=64, B=1, n=4, C=64, eps=1e-6):
    rows = [None if t is None else ctypes.byref(Rows(*t)) for t in (x, y)]
    return ra.library().rapid_norm_modulate(*rows, scale, ss, shift, hs, B, n, C, eps, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(x=(None, 0, 64)), NULL), (dict(y=(None, 0, 64)), NULL),
    (dict(scale=None), NULL), (dict(shift=None), NULL),
    (dict(B=0), SHAPE), (dict(n=0), SHAPE), (dict(C=0), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE),
    (dict(B=1 << 16, n=1 << 15), SHAPE), (dict(x=(A, 0, -64)), SHAPE), (dict(y=(3 * A, 0, 56)), SHAPE),
    (dict(B=2, x=(A, 256, 64), y=(3 * A, 248, 64)), SHAPE), (dict(B=2, x=(A, 256, 64), y=(3 * A, 256, 64), ss=-64), SHAPE),
    (dict(C=60), UNSUPPORTED), (dict(C=16392, x=(A, 0, 16392), y=(3 * A, 0, 16392)), UNSUPPORTED),
    (dict(x=(A + 2, 0, 64)), ALIGN), (dict(y=(3 * A + 8, 0, 64)), ALIGN), (dict(scale=A + 2), ALIGN), (dict(shift=A + 2), ALIGN),
    (dict(x=(A, 0, 68)), ALIGN), (dict(B=2, x=(A, 256, 64), y=(3 * A, 256, 64), hs=68), ALIGN),
    (dict(y=(A, 0, 72)), ALIAS), (dict(y=(4 * A, 0, 64)), ALIAS), (dict(y=(5 * A, 0, 64)), ALIAS),
], ids=str)
def test_modulate_refusals(kw, code):
    assert modulate(**kw) == code


def table(positions=A, tokens=4, axes=((64,),), magnitude=1.0, out=2 * A, n_axes=None):
    arr = (ra.RopeAxis * max(len(axes), 1))(*(ra.RopeAxis(*a) for a in axes)) if axes is not None else None
    n = len(axes or ()) if n_axes is None else n_axes
    return ra.library().rapid_rope_table(positions, tokens, n, arr, magnitude, out, None)


@pytest.mark.parametrize("kw,code", [
    (dict(positions=None), NULL), (dict(axes=None), NULL), (dict(out=None), NULL),
    (dict(tokens=0), SHAPE), (dict(tokens=(1 << 28) + 1), SHAPE), (dict(axes=()), SHAPE), (dict(axes=((2,),) * 9), SHAPE),
    (dict(axes=((0,),)), UNSUPPORTED), (dict(axes=((63,),)), UNSUPPORTED), (dict(axes=((24,),)), UNSUPPORTED),
    (dict(axes=((128,), (16,))), UNSUPPORTED), (dict(axes=((64, 0.0),)), UNSUPPORTED), (dict(axes=((64, float("inf")),)), UNSUPPORTED),
    (dict(axes=((64, 1e4, "linear", 0.0),)), UNSUPPORTED), (dict(axes=((64, 1e4, "ntk", float("nan")),)), UNSUPPORTED),
    (dict(axes=((2, 1e4, "ntk", 2.0), (62,))), UNSUPPORTED), (dict(axes=((64, 1e4, "by_parts", 2.0, 0.0),)), UNSUPPORTED),
    (dict(axes=((64, 1e4, "by_parts", 2.0, 64.0, 1.0, 1.0),)), UNSUPPORTED), (dict(magnitude=float("inf")), UNSUPPORTED),
    (dict(positions=A + 2), ALIGN), (dict(out=2 * A + 8), ALIGN),
], ids=str)
def test_table_refusals(kw, code):
    assert table(**kw) == code
    if "axes" not in kw:
        bad = ra.RopeAxis(64)
        bad.scaling = 4
        assert ra.library().rapid_rope_table(A, 4, 1, (ra.RopeAxis * 1)(bad), 1.0, 2 * A, None) == UNSUPPORTED


SEG = dict(q=A, k=2 * A, q_out=3 * A, k_out=4 * A, q_weight=None, k_weight=None, n=4, in_b=512, in_h=256, in_n=64, out_b=512, out_h=256, out_n=64)


def qk(segs=({},), B=1, H=2, D=64, eps=1e-6, table=6 * A, table_b=0, rot=64, layout=0, n_segments=None, norm=True):
    arr = (QkSegment * max(len(segs), 1))(*(QkSegment(*{**SEG, **s}.values()) for s in segs)) if segs is not None else None
    n = len(segs or ()) if n_segments is None else n_segments
    if norm:
        return ra.library().rapid_qk_norm_rope(arr, n, B, H, D, eps, table, table_b, rot, layout, None)
    return ra.library().rapid_rope(arr, n, B, H, D, table, table_b, rot, layout, None)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(segs=None, n_segments=1), NULL), (dict(segs=()), NULL), (dict(segs=({},) * 3), SHAPE),
    *((dict(segs=({name: None},)), NULL) for name in ("q", "k", "q_out", "k_out")),
    (dict(B=0), SHAPE), (dict(H=0), SHAPE), (dict(B=1 << 10, H=1 << 10), SHAPE), (dict(segs=({"n": 0},)), SHAPE),
    (dict(segs=({"n": (1 << 22) + 1},)), SHAPE), (dict(segs=({"n": 1 << 22}, {})), SHAPE), (dict(segs=({"in_n": -64},)), SHAPE),
    (dict(segs=({"out_n": 0},)), SHAPE), (dict(segs=({"out_h": 56},)), SHAPE), (dict(B=2, segs=({"out_b": 0},)), SHAPE),
    (dict(segs=({"in_h": 1 << 41},)), SHAPE), (dict(B=2, table_b=-4), SHAPE),
    (dict(D=96), UNSUPPORTED), (dict(rot=8), UNSUPPORTED), (dict(rot=80), UNSUPPORTED), (dict(rot=0), UNSUPPORTED), (dict(layout=2), UNSUPPORTED),
    (dict(layout=-1), UNSUPPORTED),
    *((dict(segs=({name: A + 8},)), ALIGN) for name in ("q", "k", "q_out", "k_out")),
    (dict(segs=({"in_n": 68},)), ALIGN), (dict(segs=({"out_h": 260},)), ALIGN), (dict(table=A + 8), ALIGN), (dict(B=2, table_b=6), ALIGN),
    (dict(segs=({"q_out": 4 * A},)), ALIAS), (dict(segs=({"q_out": 2 * A},)), ALIAS), (dict(segs=({"k_out": A},)), ALIAS),
    (dict(segs=({"q_out": A, "out_n": 72},)), ALIAS), (dict(segs=({"k_out": 2 * A, "in_h": 320},)), ALIAS),
], ids=str)
def test_qk_refusals(kw, code, norm):
    assert qk(**kw, norm=norm) == code


def test_qk_refusals_of_one_form():
    assert qk(table=None, norm=False) == NULL
    assert qk(eps=-1e-6) == SHAPE and qk(eps=float("nan")) == SHAPE
    assert qk(segs=({"q_weight": A + 2},)) == ALIGN and qk(segs=({"k_weight": A + 2},)) == ALIGN


def test_python_forms_take_tensors_of_the_gpu_alone():
    x = torch.zeros((1, 4, 64), dtype=torch.bfloat16)
    q = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16)
    for call in (lambda: ra.rapid_linear(x, x[0], x), lambda: ra.rapid_norm_modulate(x, x), lambda: ra.rapid_linear(1, x, x),
                 lambda: ra.rapid_rope_table(torch.zeros(4, 1, dtype=torch.int32), [ra.RopeAxis(64)], torch.zeros(4, 32, 2)),
                 lambda: ra.rapid_rope([(q, q, q, q)], torch.zeros(4, 32, 2)), lambda: ra.rapid_qk_norm_rope([(q, q, q, q)])):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ra.rapid_rope([], x), lambda: ra.rapid_rope([(q, q, q, q)], x, "other"), lambda: ra.RopeAxis(64, scaling="other")):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("kw", [
    dict(bias=3 * A), dict(gate=3 * A), dict(res=(3 * A, 0, 40)), dict(B=2, x=(A, 256, 64), y=(3 * A, 128, 32), res=(3 * A, 256, 32)),
    dict(B=2, x=(A, 256, 64), y=(3 * A, 128, 32), res=(3 * A, 0, 32)), dict(res=(3 * A, 0, 0))], ids=str)
def test_linear_outputs_that_begin_where_something_added_does(kw):
    assert linear(**kw) == ALIAS


@pytest.mark.parametrize("C,rows", [(8, 1 << 26), (2048, 1 << 26), (2056, 1 << 25), (8192, 1 << 24), (16384, 1 << 23)])
def test_rows_that_a_launch_does_not_hold(C, rows):
    for n in (rows, (1 << 31) - 257):
        assert modulate(x=(A, 0, C), y=(3 * A, 0, C), n=n, C=C) == SHAPE


def test_heads_that_a_launch_does_not_hold():
    assert qk(B=1 << 8, H=1 << 9, D=128, segs=({"n": 1 << 22, "out_b": 1 << 40, "out_n": 128, "out_h": 1 << 30, "in_n": 128},), rot=64) == SHAPE


@pytest.mark.parametrize("axis", [(64, 1e-6, "none"), (64, 1e4, "linear", 1e-6), (64, 1e-12, "ntk", 2.0)], ids=str)
def test_turns_that_cannot_be_reduced(axis):
    assert table(axes=(axis,)) == UNSUPPORTED


@pytest.mark.skipif(binding._load_native().__class__ is binding._NoNative, reason="the native calls are not built for this torch")
def test_native_forms_leave_other_tensors_to_the_python_form():
    x, q = torch.zeros((1, 4, 64), dtype=torch.bfloat16), torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16)
    positions, turns = torch.zeros(4, 1, dtype=torch.int32), torch.zeros(4, 32, 2)
    native = binding._load_native()
    assert native.linear(x, x[0], x, None, "none", None, None, None) is None
    assert native.modulate(x, x, None, None, 1e-6) is None
    assert native.table(positions, [ra.RopeAxis(64)], turns, 1.0) is None
    assert native.qk_norm_rope([(q, q, q, q)], None, turns, "interleaved", 1e-6) is None
    assert native.rope([(q, q, q, q)], None, turns, "half") is None
