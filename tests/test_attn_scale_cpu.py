"""Scales that pc_attn refuses on the host."""
import pytest

import paper_2608_01657_amd as P
from test_pages_cpu import _attn, _pool


@pytest.mark.parametrize("scale", [3.4e38, 2.4e38, -1e-30, float("-inf")])
def test_scales_that_leave_the_range(scale):
    """The scale is taken in powers of two: log2(e) times it has to be a finite float too."""
    assert _attn(_pool(), scale=scale) == P.PC_EINVAL
    assert "scale" in P.pc_last_error()
