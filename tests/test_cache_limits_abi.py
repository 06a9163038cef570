"""Arguments at the limits of the 4-bit cache's entry points.  CPU only: every call fails validation or launches nothing."""
import pytest

from tests.test_cache_abi import INVALID, WORKSPACE, attend, cdesc, lib  # noqa: F401


@pytest.mark.parametrize("scale", [2.4e38, 2.9e38, 3.4e38])
def test_scale_whose_product_is_no_number(lib, scale):  # noqa: F811
    """Every exponent would be infinite or NaN."""
    assert attend(lib, cdesc(), scale=scale) == INVALID


@pytest.mark.parametrize("scale", [1e-45, 1.0, 2.3e38])
def test_scales_that_are_taken(lib, scale):  # noqa: F811
    # (as far as the workspace, which is missing)
    assert attend(lib, cdesc(), scale=scale, ws=None) == WORKSPACE
