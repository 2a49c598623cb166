"""Host-only checks of calls that the operators around the attention have to refuse, at the limits of their sizes and strides and
where outputs would be written twice."""
import pytest

from test_layer_abi import A, SHAPE, linear, modulate


@pytest.mark.parametrize("B,stride_b", [((1 << 23) + 1, 1 << 40), ((1 << 24) + 1, 1 << 40), ((1 << 25) + 1, 3 << 38)], ids=str)
@pytest.mark.parametrize("n", [2, 3])
def test_rows_that_share_elements_in_far_samples(B, stride_b, n):
    """Rows of an output 16 elements apart and longer than that, samples so far apart that their distance by their number passes
    64 bits."""
    assert linear(B=B, n=n, x=(A, 128, 64), y=(3 * A, stride_b, 16)) == SHAPE
    assert modulate(B=B, n=n, x=(A, 256, 64), y=(3 * A, stride_b, 16)) == SHAPE


def test_samples_within_the_distance_of_rows_are_no_overlap():
    """Samples of a token side by side pass this check: the next one (alignment) is what refuses these calls."""
    from test_layer_abi import ALIGN
    assert linear(B=3, x=(A + 8, 64, 192), y=(3 * A, 32, 96)) == ALIGN
    assert modulate(B=3, x=(A + 8, 64, 192), y=(3 * A, 64, 192)) == ALIGN
    assert linear(B=3, x=(A + 8, 64, 192), y=(3 * A, 32, 95)) == SHAPE and modulate(B=3, x=(A + 8, 64, 192), y=(3 * A, 64, 184)) == SHAPE
