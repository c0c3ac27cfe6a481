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


def test_an_empty_list_of_groups():
    from tests.seqcache import filled, i32
    c, _ = filled([40, 7], 2, 64, torch.bfloat16, 1)
    q = torch.randn(2, 4, 64, device="cuda").bfloat16()
    for max_len in (0, 40):
        want = c.prefix_attention(0, q, i32([0, 1]), max_len=max_len)
        got = c.prefix_attention(0, q, i32([0, 1]), i32([0]), i32([]), max_len=max_len)
        assert torch.equal(got, want)


def test_one_row_of_any_stride():
    from tests.seqcache import filled, i32
    c, _ = filled([40], 2, 64, torch.bfloat16, 1)
    q = torch.randn(4 * 64, device="cuda").bfloat16()
    want = c.prompt_attention(0, q.view(1, 4, 64), i32([0]), i32([0, 1]))
    for stride in (1, 4 * 64 + 1):
        got = c.prompt_attention(0, q.as_strided((1, 4, 64), (stride, 64, 1)), i32([0]), i32([0, 1]))
        assert torch.equal(got, want)


def test_the_output_is_not_the_input():
    from paper_2605_30852_amd import binding as B
    from tests.seqcache import filled, i32
    c, _ = filled([40], 2, 64, torch.bfloat16, 1)
    q = torch.randn(1, 4, 64, device="cuda").bfloat16()
    keep = q.clone()
    for max_len in (0, 40):
        with pytest.raises(B.SPDError, match="out must not be q"):
            c.prompt_attention(0, q, i32([0]), i32([0, 1]), out=q, max_len=max_len)
        with pytest.raises(B.SPDError, match="out must not be q"):
            c.prefix_attention(0, q, i32([0]), out=q, max_len=max_len)
    assert torch.equal(q, keep)


@pytest.mark.parametrize("max_len", [0, 300])
def test_a_sequence_named_twice_is_read_twice(max_len):
    from tests.seqcache import filled, i32
    c, _ = filled([300, 20], 2, 128, torch.float32, 2)
    q = torch.randn(33, 6, 128, device="cuda")
    out = c.prompt_attention(0, torch.cat((q, q[:5], q)), i32([0, 1, 0]), i32([0, 33, 38, 71]), max_len=max_len)
    assert torch.equal(out[:33], out[38:])
    rows = c.prefix_attention(0, torch.cat((q[:1], q[:1], q[:1])), i32([0, 0, 0]), i32([0, 3]), i32([300]), max_len=max_len)
    assert torch.equal(rows[0], rows[1]) and torch.equal(rows[0], rows[2])


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("f32", "f32")], ids="-".join)
def test_hundreds_of_kv_heads(types):
    from tests.test_gpu_seq_attention import run_prefix, run_prompt
    heads = (600, 600, 64)
    run_prompt([3, 20], [300, 1], heads, types, seed=6)
    run_prefix([3, 1], [290, 0], [300, 291, 310, 5], heads, types, seed=6)


@pytest.mark.parametrize("heads", [(8, 2, 128), (6, 2, 64), (16, 1, 128), (3, 3, 64)], ids=str)
def test_seventeen_to_thirty_two_queries_of_an_fp32_cache(heads):
    """Two sets of 16 queries a piece, split over long caches and not, with a prefix shared by as many."""
    from tests.test_gpu_seq_attention import run_prefix, run_prompt
    G = heads[0] // heads[1]
    few, most = 16 // G + 1, 32 // G
    for seed, cached in enumerate(([0, 3000, 17, 1200], [31, 255, 256, 700])):
        run_prompt([few, most, most, few], cached, heads, ("f32", "f32"), seed=seed, tail=1, pad=4)
    lens = [1500 + 7 * i for i in range(most)]
    run_prefix([most], [1490], lens, heads, ("f32", "f32"), seed=3)


def test_values_that_are_not_finite_in_two_sets_of_queries():
    from tests.seqcache import filled, i32
    n = 8
    for where, what in ((1, float("inf")), (1, float("nan")), (0, float("nan"))):
        c, _ = filled([600], 2, 64, torch.float32, 3)
        page = int(c.page_table[0, 37])
        c.kv[0, page, where, 0, 4, 7] = what  # key 596 of KV head 0: rows 4 and up attend it
        q = torch.randn(n, 8, 64, generator=torch.Generator().manual_seed(1)).cuda()
        out = c.prompt_attention(0, q, i32([0]), i32([0, n]))
        assert torch.isfinite(out[:4]).all() and torch.isfinite(out[:, 4:]).all()
        assert not torch.isfinite(out[4:, :4, 7]).any()
        if where == 0:
            assert torch.isnan(out[4:, :4]).all()
