"""Arguments of the target's operators that no list of tests/test_target_abi.py has (CPU)."""

import pytest

from test_target_abi import INVALID, attend

from paper_2607_04244_amd import qlin


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_a_scale_whose_exponents_have_no_factor_is_refused(scale):
    """scale log2(e), the factor of the base-2 exponents, is no finite number."""
    assert attend(scale=scale) == INVALID and "scale" in qlin.last_error()
    assert attend(scale=2.3e38, ws=None, wb=0, splits=3) == INVALID and "workspace" in qlin.last_error()
