"""The packed cache's and the rotation's host code at the limits of what its calls take.  No GPU."""
import pytest

from paper_2607_20125_b200 import packed


@pytest.mark.parametrize("scale", [1e-60, -1e-60, 2.0 ** -151, 5e-324])
def test_a_scale_that_a_c_float_cannot_hold_is_not_taken_for_the_default(scale):
    with pytest.raises(ValueError, match="softmax_scale"):
        packed.PackedCache(4, 64, 100, softmax_scale=scale)


@pytest.mark.parametrize("scale", [1e-20, 2.0 ** -41, 2.0 ** 41, -1.0, 1e60, float("nan"), float("inf")])
def test_scales_out_of_range_are_refused(scale):
    with pytest.raises(packed.HeadCastError, match="softmax_scale"):
        packed.PackedCache(4, 64, 100, softmax_scale=scale)
