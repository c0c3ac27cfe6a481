"""The ways a call on a cache of several sequences can go: without a plan (short calls), with more sequences, tiles or
memory than the plan keeps at hand, on other streams, twice at once, and the same every time."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]


def dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("heads", [(8, 2, 128), (5, 1, 64), (32, 2, 128), (6, 6, 64)], ids=str)
@pytest.mark.parametrize("max_len", [65, 512])
def test_short_prompts(heads, types, max_len):
    from tests.test_gpu_seq_attention import run_prompt
    run_prompt([1, 17, 0, 45, 16, 2], [0, 3, 9, 20, 31, 63], heads, types, seed=2, tail=2, max_len=max_len, pad=8)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_short_prompts_that_are_longer_than_said(types):
    from tests.test_gpu_seq_attention import run_prompt
    run_prompt([3, 40], [700, 560], (8, 2, 128), types, seed=3, max_len=512)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("heads", [(8, 2, 128), (3, 1, 64), (16, 1, 128)], ids=str)
def test_decode_rows_that_share_nothing(heads, types):
    from tests.test_gpu_seq_attention import run_prefix
    for max_len in (400, 100, 0):
        run_prefix([1] * 7, [0] * 7, [1, 0, 16, 31, 33, 400, 129], heads, types, seed=4, max_len=max_len, use_groups=False)


def small_cache(n_seqs, most, hkv, dh, seed):
    """Many short sequences, filled on the GPU."""
    from paper_2605_30852_amd.cache import PagedCache
    g = torch.Generator(device="cuda").manual_seed(seed)
    lens = torch.randint(1, most + 1, (n_seqs,), generator=g, device="cuda", dtype=torch.int32)
    width = (most + 15) // 16
    ids = torch.randperm(n_seqs * width, generator=g, device="cuda").int().view(n_seqs, width)
    kv = torch.empty(1, n_seqs * width, 2, hkv, 16, dh, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    return PagedCache(kv, ids, lens), lens.tolist()


def keys_of(cache, s, n):
    ids = cache.page_table[s, :(n + 15) // 16].long()
    return cache.kv[0, ids].permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :n]


def test_more_sequences_than_the_plan_keeps():
    """5000 sequences of one to five new rows: past the 4096 that the plan holds in LDS."""
    from tests.seqcache import attend, check, i32
    n, hq, hkv, dh = 5000, 2, 1, 64
    cache, lens = small_cache(n, 40, hkv, dh, 1)
    rng = random.Random(2)
    rows = [min(rng.choice([0, 1, 1, 2, 5]), lens[s]) for s in range(n)]
    cu = [0]
    for r in rows:
        cu.append(cu[-1] + r)
    q = (1.5 * torch.randn(cu[-1], hq, dh, device="cuda")).bfloat16()
    out = cache.prompt_attention(0, q, i32(list(range(n))), i32(cu))
    assert torch.isfinite(out).all()
    for s in [0, 1, 4095, 4096, 4097, n - 1] + rng.sample(range(n), 60):
        k, v = keys_of(cache, s, lens[s])
        want, mag = attend(q[cu[s]:cu[s + 1]], k, v, [lens[s] - rows[s] + r + 1 for r in range(rows[s])])
        check(out[cu[s]:cu[s + 1]], want, mag, ("bf16", s))


def test_more_groups_than_the_plan_keeps():
    """2048 groups of two rows: more tiles than the 1024 whose records the plan holds in LDS."""
    from tests.seqcache import agree, attend, check, i32
    n, hq, hkv, dh = 4096, 2, 1, 64
    cache, lens = small_cache(n, 60, hkv, dh, 5)
    rng = random.Random(6)
    prefix = [rng.choice([0, 1, 16, 20, 48, 70]) for _ in range(n // 2)]
    for j, p in enumerate(prefix):
        agree(cache, 2 * j, 2 * j + 1, min(p, lens[2 * j], lens[2 * j + 1]))
    q = (1.5 * torch.randn(n, hq, dh, device="cuda")).bfloat16()
    out = cache.prefix_attention(0, q, i32(list(range(n))), i32(list(range(0, n + 1, 2))), i32(prefix))
    assert torch.isfinite(out).all()
    for s in [0, 1, 2046, 2047, 2048, 2049, n - 2, n - 1] + rng.sample(range(n), 80):
        first = s - s % 2
        m = min(prefix[s // 2], lens[first], lens[s])
        a, b = keys_of(cache, first, lens[first]), keys_of(cache, s, lens[s])
        x = torch.cat([a[:, :, :m], b[:, :, m:]], 2)
        want, mag = attend(q[s:s + 1], x[0], x[1], [lens[s]])
        check(out[s:s + 1], want, mag, ("bf16", s))


def test_a_pool_past_four_gigabytes():
    """Offsets past 32 bits, of the page and of the layer: attention, new rows and copies."""
    from paper_2605_30852_amd.cache import PagedCache
    from tests.seqcache import attend, check, i32
    pages, hkv, dh = 36000, 8, 128  # 64 KB a page: 2.4 GB a layer
    kv = torch.empty(2, pages, 2, hkv, 16, dh, dtype=torch.bfloat16, device="cuda")
    top = list(range(pages - 4, pages))
    kv[:, top] = torch.randn(2, 4, 2, hkv, 16, dh, device="cuda").bfloat16()
    refs = torch.ones(pages, dtype=torch.int32, device="cuda")
    refs[pages - 1] = 0
    refs[pages - 2] = 2
    c = PagedCache(kv, i32([[pages - 4, pages - 3, -1], [pages - 4, pages - 2, -1]]), i32([32, 29]), refs)
    q = (1.5 * torch.randn(32, 16, dh, device="cuda")).bfloat16()
    out = c.prompt_attention(1, q, i32([0]), i32([0, 32]))
    x = kv[1, top[:2]].permute(1, 2, 0, 3, 4).flatten(2, 3)
    want, mag = attend(q, x[0], x[1], list(range(1, 33)))
    check(out, want, mag, ("bf16",))
    assert c.reserve(i32([1]), i32([1])).item() == 0  # the shared last page goes to the only free one
    assert c.page_table[1].tolist() == [pages - 4, pages - 1, -1] and torch.equal(kv[:, pages - 1], kv[:, pages - 2])
    k = torch.randn(1, hkv, dh, device="cuda").bfloat16()
    c.append(1, k, k + 1, i32([1]), i32([0, 1]))
    assert torch.equal(kv[1, pages - 1, 0, :, 13], k[0]) and torch.equal(kv[1, pages - 1, 1, :, 13], k[0] + 1)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_the_same_bits_every_time_on_any_stream(types):
    """Calls repeated, on other streams and at once; a sequence is named twice."""
    from tests.seqcache import filled, i32
    lens = [1300, 40, 700, 90]
    c, _ = filled(lens, 2, 128, dt(types[1]), 4)
    q = torch.randn(70, 8, 128, generator=torch.Generator().manual_seed(2)).to(dt(types[0])).cuda()
    seqs, cu = i32([0, 2, 1]), i32([0, 5, 60, 70])
    groups, prefix, dec = i32([0, 2, 5]), i32([600, 30]), i32([0, 2, 1, 3, 3])

    def both():
        return c.prompt_attention(0, q, seqs, cu), c.prefix_attention(0, q[:5], dec, groups, prefix)

    a = both()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(5):
        outs = []
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                outs.append(both())
        torch.cuda.synchronize()
        for o in outs:
            assert torch.equal(o[0], a[0]) and torch.equal(o[1], a[1])


def test_batches_without_rows():
    from tests.seqcache import filled, i32
    c, _ = filled([20, 0, 5], 2, 64, torch.bfloat16, 1)
    q = torch.randn(4, 4, 64, device="cuda").bfloat16()
    for max_len in (0, 30):
        out = torch.full_like(q, 7.0)
        c.prompt_attention(0, q, i32([0, 1, 2]), i32([0, 0, 0, 0]), out=out, max_len=max_len)
        assert (out == 7.0).all()
        out = c.prompt_attention(0, q, i32([1]), i32([0, 4]), max_len=max_len)  # rows of a sequence without keys
        assert (out == 0).all()
        c.prompt_attention(0, q[:0], i32([0]), i32([0, 0]), max_len=max_len)
        out = c.prefix_attention(0, q[:2], i32([1, 1]), max_len=max_len)
        assert (out == 0).all()
    before = c.kv.clone()
    c.append(0, q[:, :2], q[:, :2], i32([1]), i32([0, 4]))  # positions before the first
    torch.cuda.synchronize()
    assert torch.equal(c.kv.view(torch.int16), before.view(torch.int16))


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_values_that_are_not_finite_in_short_calls(types):
    """The plain pass of pieces of few queries: an infinite value behind a row's position, NaN in a key."""
    from tests.seqcache import filled, i32
    n = 60
    for where, what in ((1, float("inf")), (1, float("nan")), (0, float("nan"))):
        c, kv = filled([n], 2, 64, dt(types[1]), 3)
        page = int(c.page_table[0, 2])
        c.kv[0, page, where, 0, 8, 7] = what  # key 40 of KV head 0
        q = torch.randn(n, 4, 64, generator=torch.Generator().manual_seed(1)).to(dt(types[0])).cuda()
        out = c.prompt_attention(0, q, i32([0]), i32([0, n]), max_len=n)
        assert torch.isfinite(out[:40]).all() and torch.isfinite(out[:, 2:]).all()
        assert not torch.isfinite(out[40:, :2, 7]).any()
        if where == 1:
            rest = torch.ones(64, dtype=torch.bool)
            rest[7] = False
            assert torch.isfinite(out[40:, :2][:, :, rest]).all()
        else:
            assert torch.isnan(out[40:, :2]).all()
        one = c.prefix_attention(0, q[-1:], i32([0]), max_len=n)
        assert torch.equal(torch.isnan(one), torch.isnan(out[-1:])) and torch.equal(torch.isinf(one), torch.isinf(out[-1:]))


def test_python_refusals():
    from paper_2605_30852_amd import binding as B
    from paper_2605_30852_amd.cache import PagedCache
    from tests.seqcache import filled, i32
    c, _ = filled([20, 5], 2, 64, torch.bfloat16, 1)
    q = torch.randn(3, 4, 64, device="cuda").bfloat16()
    s, cu = i32([0]), i32([0, 3])
    good = c.prompt_attention(0, q, s, cu)
    for bad in (dict(q=q.float().double()), dict(q=q[:, :, ::2]), dict(q=q.transpose(0, 1)), dict(q=q.cpu()), dict(q=q[..., :32]),
                dict(seqs=s.long()), dict(seqs=s.cpu()), dict(cu_rows=i32([0])), dict(out=torch.empty(2, 4, 64, device="cuda").bfloat16())):
        with pytest.raises(ValueError):
            c.prompt_attention(0, **{**dict(q=q, seqs=s, cu_rows=cu), **bad})
    for bad in (dict(q=q[:, :3]), dict(layer=1), dict(max_len=-1)):
        with pytest.raises(B.SPDError):
            c.prompt_attention(**{**dict(layer=0, q=q, seqs=s, cu_rows=cu), **bad})
    with pytest.raises(ValueError):
        c.prefix_attention(0, q[:1], s, cu_groups=i32([0, 1]))
    with pytest.raises(ValueError):
        c.append(0, q[:, :2], q[:, :2], s, cu, q_out=q)
    with pytest.raises(ValueError):
        c.reserve(s, i32([1, 2]))
    with pytest.raises(B.SPDError):
        PagedCache(c.kv, c.page_table, c.lens).reserve(s, s)  # no counts
    with pytest.raises(ValueError):
        PagedCache(c.kv[:, ::2], c.page_table, c.lens)
    assert torch.equal(good, c.prompt_attention(0, q, s, cu))
