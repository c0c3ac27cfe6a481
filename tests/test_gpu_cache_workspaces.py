"""Memory that the calls on a large pool's pages take, and a truncate without a workspace."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def requested(call):
    key = "requested_bytes.all.allocated"
    before = torch.cuda.memory_stats()[key]
    out = call()
    return torch.cuda.memory_stats()[key] - before, out


def test_truncate_and_fork_of_a_large_pool():
    from paper_2605_30852_amd import binding as B
    from paper_2605_30852_amd.cache import PagedCache
    from tests.seqcache import i32
    c = PagedCache.empty(1, 200000, 1, 64, 100, 300)
    who, add = i32([0, 1]), i32([300, 17])
    assert c.reserve(who, add).item() == 0
    for n in (2, 90):
        src, dst, keep, none = i32([0] * n), i32(list(range(2, n + 2))), i32([290] * n), i32([0] * n)
        took, st = requested(lambda: c.fork(src, dst, keep))
        assert st.item() == 0 and took < 1024 and c.refs[0].item() == n + 1
        took, st = requested(lambda: c.truncate(dst, none))
        assert st.item() == 0 and took < 1024 and c.refs[0].item() == 1
    keep = i32([3, 0])
    word = i32([-1])
    B.spd_cache_truncate(c.c, who.data_ptr(), keep.data_ptr(), 2, word.data_ptr(), None, 0, torch.cuda.current_stream().cuda_stream)
    assert word.item() == 0 and c.lens[:2].tolist() == [3, 0] and int(c.refs.sum()) == 1
    took, live = requested(c.compact)
    assert live.item() == 1 and 12 * 200000 <= took < 12 * 200000 + 4096
