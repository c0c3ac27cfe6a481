"""What the calls that change a cache's pages ask for as workspace, on the host (the pointers here are never dereferenced: a call
that passes its checks ends at the launch, for want of a GPU)."""
import pytest

from paper_2605_30852_amd import binding as B
from tests.test_cache_refusals import cache, refused

PAGES = 3_000_000


def launched(call, *a):
    import torch
    if torch.cuda.is_available():
        pytest.skip("would launch on pointers that are none")
    with pytest.raises(B.SPDError) as e:
        call(*a)
    assert e.value.status == B.SPD_E_HIP, e.value


def test_truncate_needs_none():
    launched(B.spd_cache_truncate, cache(num_pages=PAGES), 4, 8, 2, 16, 0, 0, 0)


def test_fork_needs_a_header():
    c = cache(num_pages=PAGES)
    launched(B.spd_cache_fork, c, 4, 8, 12, 2, 16, 256, 256, 0)
    refused(B.spd_cache_fork, c, 4, 8, 12, 2, 16, 0, 256, 0)
    refused(B.spd_cache_fork, c, 4, 8, 12, 2, 16, 128, 256, 0)
    refused(B.spd_cache_fork, c, 4, 8, 12, 2, 16, 256, 16, 0, code=B.SPD_E_CAPACITY)


def test_reserve_and_compact_need_their_lists():
    c = cache(num_pages=PAGES)
    for n in (1, 4):
        need = B.spd_cache_workspace(c, n)
        assert 12 * PAGES <= need <= 12 * PAGES + 1024
        launched(B.spd_cache_compact, c, 4, 256, need, 0)
        refused(B.spd_cache_compact, c, 4, 256, 12 * PAGES, 0, code=B.SPD_E_CAPACITY)
        launched(B.spd_cache_reserve, c, 4, 8, n, 12, 256, 4 * PAGES + 256, 0)
        refused(B.spd_cache_reserve, c, 4, 8, n, 12, 256, 4 * PAGES, 0, code=B.SPD_E_CAPACITY)
    many = cache(num_pages=3, max_seqs=60000)  # more entries than pages
    need = B.spd_cache_workspace(many, 60000)
    launched(B.spd_cache_reserve, many, 4, 8, 60000, 12, 256, need, 0)
    refused(B.spd_cache_reserve, many, 4, 8, 60000, 12, 256, 16 * 60000, 0, code=B.SPD_E_CAPACITY)
