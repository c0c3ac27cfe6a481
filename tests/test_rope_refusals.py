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


def test_numbers_of_more_bits_than_the_call_takes():
    """ctypes cuts them without a word: 2^32 + 64 dims were 64 with as many zeros behind them."""
    torch = pytest.importorskip("torch")
    from paper_2605_30852_amd.rope import RopeScaling, rope_frequencies, rope_table
    freq = rope_frequencies(64, 1e4)
    for dims in ((1 << 32) + 64, -(1 << 32) + 64):
        with pytest.raises(ValueError, match="dims"):
            rope_frequencies(dims, 1e4)
    with pytest.raises(ValueError, match="original"):
        rope_frequencies(64, 1e4, RopeScaling("parts", 4.0, original=(1 << 32) + 4096))
    with pytest.raises(ValueError, match="positions"):
        rope_table(freq, (1 << 32) + 5, out=(torch.empty(0), torch.empty(0)))
    for first in (1 << 64, -(1 << 64), (1 << 30) + 1):
        with pytest.raises(ValueError, match="first"):
            rope_table(freq, 5, first=first, out=(torch.empty(0), torch.empty(0)))


@pytest.mark.parametrize("cos, sin", [(1 << 20, 1 << 20), (1 << 20, (1 << 20) + 16), ((1 << 20) + 32, 1 << 20)])
def test_tables_that_overlap(cos, sin):
    """Each would hold some of the other's values. (Addresses that the call would launch with: no GPU is here, and that is an error of
    another kind.)"""
    with pytest.raises(B.SPDError) as e:
        B.spd_rope_table((ct.c_double * 4)(1.0, 0.5, 0.1, 0.0), 4, 0, 3, 1.0, cos, sin, 0)
    assert e.value.status == B.SPD_E_INVAL
