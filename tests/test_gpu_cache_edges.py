"""Calls on a cache of several sequences that are allowed and unusual: more sequences than a launch has workgroups,
no groups at all, one row of any stride, a sequence named twice, hundreds of KV heads."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_truncate_of_more_sequences_than_workgroups():
    from tests.seqcache import i32
    from tests.test_gpu_cache_pages import make, same
    n = 1700
    c, m, kv0 = make(4 * n, n, 5, layers=1, hkv=1)
    rng = random.Random(1)
    seqs = rng.sample(range(n), n)
    add = [rng.randint(0, 64) for _ in seqs]
    same(c, m, kv0, c.reserve(i32(seqs), i32(add)), m.reserve(seqs, add), "grow")
    keep = [rng.choice([0, 1, 16, 31, 200]) for _ in seqs]
    for last, want in ((seqs[0], 3), (-1, 3), (n, 3)):
        bad = seqs[:-1] + [last]
        assert m.truncate(bad, keep) == want
        same(c, m, kv0, c.truncate(i32(bad), i32(keep)), want, last)
    bad = keep[:-1] + [-1]
    same(c, m, kv0, c.truncate(i32(seqs), i32(bad)), m.truncate(seqs, bad), "a length")
    same(c, m, kv0, c.truncate(i32(seqs), i32(keep)), m.truncate(seqs, keep), "cut")
