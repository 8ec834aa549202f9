"""Scales of the attention's scores that the kernels' own, times log2(e), has no binary32 number for: refused before any device work (they made every score NaN)."""
import math

import pytest

from paper_2410_20650_amd import binding as nz
from test_more_operator_arguments import attention

MOST = 2.0 ** 128 * (1 - 2.0 ** -24) / 1.4426950408889634     # the largest float32 over log2(e)


@pytest.mark.parametrize("scale", [MOST * (1 + 2.0 ** -20), 2.4e38, 3.4e38, math.inf])
def test_scales_that_leave_binary32(scale):
    assert attention(scale=scale) == nz.EINVAL
