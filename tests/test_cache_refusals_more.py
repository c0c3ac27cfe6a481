"""Further refusals of the calls on a cache of several sequences, on the host (the pointers here are never dereferenced)."""
import pytest

from paper_2605_30852_amd import binding as B
from tests.test_cache_refusals import append, refused


@pytest.mark.parametrize("bad", [dict(q_out=48, q_out_stride=2048), dict(q=64, q_stride=1032)], ids=str)
def test_append_in_place_between_other_strides(bad):
    """A row written where another row is still to be read."""
    refused(append, **bad)
    append(rows=0, **bad)

