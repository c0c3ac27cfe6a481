"""What the rotary calls refuse beside the arguments of test_rule_refusals: on the host, before anything is launched."""
import ctypes as ct

import pytest

from paper_2605_30852_amd import binding as B
from tests.test_cache_refusals import refused


@pytest.mark.parametrize("kind, factor, base", [(B.SPD_ROPE_BASE, 1e300, 1e30), (B.SPD_ROPE_BASE, 1e-300, 1.5), (B.SPD_ROPE_LINEAR, 5e-324, 1e4),
                                                (B.SPD_ROPE_PARTS, 5e-324, 1e4)])
def test_scalings_that_leave_the_range(kind, factor, base):
    """Their frequencies came out as 0 or as infinities."""
    refused(B.spd_rope_frequencies, 64, base, B.spd_rope_scaling(kind, 4096, factor, 1.0, 32.0))
