"""Scales of the paged cache's attention that the host refuses.  No GPU."""
import pytest

import paper_2502_00937_amd as V
from test_pages_refusals import attend


@pytest.mark.parametrize("scale", [2.5e38, -3.4e38, float("inf"), float("-inf"), float("nan")])
def test_scales_that_the_exponent_does_not_hold(scale):
    """Exponentials are powers of two: the scale times log2 e has to be a number."""
    assert attend(V.load_library(), scale=scale) == -1
    assert b"scale" in V.load_library().vit_last_error()


@pytest.mark.parametrize("scale", [2.3e38, -2.3e38, 1e-45, 0.0])
def test_scales_that_it_does(scale):
    assert attend(V.load_library(), scale=scale, rows=0) == 0
