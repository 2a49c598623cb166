"""Host-only checks of calls that the operators around the attention have to refuse, at the limits of their sizes and strides and
where outputs would be written twice."""
import pytest

from test_layer_abi import A, ALIAS, ALIGN, SHAPE, linear, modulate, qk


@pytest.mark.parametrize("B,stride_b", [((1 << 23) + 1, 1 << 40), ((1 << 24) + 1, 1 << 40), ((1 << 25) + 1, 3 << 38)], ids=str)
@pytest.mark.parametrize("n", [2, 3])
def test_rows_that_share_elements_in_far_samples(B, stride_b, n):
    """Rows of an output 16 elements apart and longer than that, samples so far apart that their distance by their number passes
    64 bits."""
    assert linear(B=B, n=n, x=(A, 128, 64), y=(3 * A, stride_b, 16)) == SHAPE
    assert modulate(B=B, n=n, x=(A, 256, 64), y=(3 * A, stride_b, 16)) == SHAPE


def test_samples_within_the_distance_of_rows_are_no_overlap():
    """Samples of a token side by side pass this check: the next one (alignment) is what refuses these calls."""
    assert linear(B=3, x=(A + 8, 64, 192), y=(3 * A, 32, 96)) == ALIGN
    assert modulate(B=3, x=(A + 8, 64, 192), y=(3 * A, 64, 192)) == ALIGN
    assert linear(B=3, x=(A + 8, 64, 192), y=(3 * A, 32, 95)) == SHAPE and modulate(B=3, x=(A + 8, 64, 192), y=(3 * A, 64, 184)) == SHAPE


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("out", [
    dict(out_h=64), dict(out_h=256, out_n=256), dict(out_h=192), dict(out_n=72), dict(out_b=448), dict(out_b=128, out_h=512, out_n=64),
    dict(out_h=64, out_n=64), dict(out_b=64, out_h=256, out_n=72)], ids=str)
def test_rows_of_queries_and_keys_that_share_elements(out, norm):
    """(B = H = 2, n = 4, D = 64: whole at strides 512, 256, 64)"""
    assert qk(B=2, segs=(out,), norm=norm) == SHAPE
    assert qk(B=2, segs=({}, dict(q=11 * A, k=12 * A, q_out=13 * A, k_out=14 * A, **out)), norm=norm) == SHAPE


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("out", [
    dict(out_b=512, out_h=64, out_n=128), dict(out_b=1536, out_h=64, out_n=384), dict(out_b=64, out_h=128, out_n=256),
    dict(out_b=128, out_h=1024, out_n=256), dict(out_b=64, out_h=512, out_n=128), dict(out_b=520, out_h=264, out_n=64)], ids=str)
def test_rows_of_queries_and_keys_in_any_order_are_apart(out, norm):
    """The check of the table's alignment, behind the one of the rows, is what refuses these calls."""
    assert qk(B=2, segs=(out,), table=6 * A + 8, norm=norm) == ALIGN


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("name,at", [("q_out", 1), ("q_out", 2), ("q_out", 3), ("q_out", 4), ("k_out", 1), ("k_out", 2), ("k_out", 3), ("k_out", 4)])
@pytest.mark.parametrize("which", [0, 1])
def test_outputs_that_begin_where_a_tensor_of_the_other_segment_does(which, name, at, norm):
    """(the first segment's tensors at A, 2 A, 3 A and 4 A)"""
    other = dict(q=11 * A, k=12 * A, q_out=13 * A, k_out=14 * A)
    segs = ({}, {**other, name: at * A})
    assert qk(segs=segs[::-1] if which else segs, norm=norm) == ALIAS


def test_workspaces_of_sizes_beyond_32_bits():
    import paper_2509_22323_amd as ra
    assert ra.rapid_linear_workspace_bytes(300, 320, 4096) > 0
    for size in ((300 + (1 << 32), 320, 4096), (300, 320 + (1 << 32), 4096), (300, 320, 4096 + (1 << 32)), (300, 320, 4096 + (1 << 31))):
        assert ra.rapid_linear_workspace_bytes(*size) == 0


def test_strides_at_their_limits():
    """Of a row 2^22, of a sample and of its vectors 2^40; calls within them are refused for their alignment, behind this check."""
    wide = dict(B=2, x=(A, 256, 64), y=(3 * A, 128, 32))
    assert linear(**{**wide, "y": (3 * A + 1, 1 << 40, 1 << 22)}) == ALIGN
    assert linear(**{**wide, "y": (3 * A + 1, (1 << 40) + 1, 32)}) == SHAPE and linear(**{**wide, "y": (3 * A + 1, 1 << 40, (1 << 22) + 1)}) == SHAPE
    assert linear(**wide, res=(A + 1, 1 << 40, 0)) == ALIGN and linear(**wide, res=(A + 1, (1 << 40) + 1, 0)) == SHAPE
    assert linear(**wide, gate=A + 1, gs=1 << 40) == ALIGN and linear(**wide, gate=A + 1, gs=(1 << 40) + 1) == SHAPE
    rows = dict(B=2, x=(A + 2, 1 << 40, 1 << 22), y=(3 * A, 1 << 40, 1 << 22), ss=1 << 40, hs=1 << 40)
    assert modulate(**rows) == ALIGN
    for far in (dict(x=(A + 2, (1 << 40) + 8, 64)), dict(x=(A + 2, 256, (1 << 22) + 8)), dict(y=(3 * A, (1 << 40) + 8, 64)), dict(ss=(1 << 40) + 8),
                dict(hs=(1 << 40) + 8)):
        assert modulate(**{**rows, **far}) == SHAPE
