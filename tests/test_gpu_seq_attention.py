"""Attention over a cache of several sequences against 64 bits: packed causal rows, and decode rows of groups that
share a prefix."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]
HEADS = [(8, 2, 128), (4, 4, 64), (6, 2, 64), (16, 1, 128), (5, 1, 128), (16, 2, 64)]


def dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def run_prompt(rows, cached, heads, types, seed=0, tail=0, max_len=0, pad=0):
    """rows[i] new rows behind cached[i] keys, in slots of another order; `tail` rows behind the last sequence, which stay
    as they are; `pad`: elements between the rows."""
    from tests.seqcache import attend, check, filled, i32
    hq, hkv, dh = heads
    rng = random.Random(seed)
    n = len(rows)
    slots = rng.sample(range(n), n)
    lens = [0] * n
    for i, s in enumerate(slots):
        lens[s] = rows[i] + cached[i]
    cache, kv = filled(lens, hkv, dh, dt(types[1]), seed)
    cu = [0]
    for r in rows:
        cu.append(cu[-1] + r)
    total = cu[-1] + tail
    g = torch.Generator().manual_seed(seed + 1)
    wide = (1.5 * torch.randn(total, hq * dh + pad, generator=g)).to(dt(types[0])).cuda()
    q = wide[:, :hq * dh].unflatten(1, (hq, dh))
    out = torch.full((total, hq * dh + pad), 7.0, dtype=dt(types[0]), device="cuda")
    print(f"[prompt {types} {heads} rows {rows} cached {cached}]", flush=True)
    cache.prompt_attention(0, q, i32(slots), i32(cu), out=out[:, :hq * dh].unflatten(1, (hq, dh)), max_len=max_len)
    torch.cuda.synchronize()
    for i, s in enumerate(slots):
        a, b = cu[i], cu[i + 1]
        limits = [cached[i] + r + 1 for r in range(rows[i])]
        want, mag = attend(q[a:b], kv[s][0, 0], kv[s][0, 1], limits)
        check(out[a:b, :hq * dh].unflatten(1, (hq, dh)), want, mag, (types[0], "sequence", i))
    assert (out[cu[-1]:] == 7.0).all() and (out[:, hq * dh:] == 7.0).all()


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_ragged_prompts(heads, types):
    run_prompt([1, 2, 17, 0, 64, 65, 33], [0, 15, 100, 5, 0, 1, 31], heads, types, tail=3)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("heads", [(8, 2, 128), (3, 1, 64)], ids=str)
def test_long_prompts(heads, types):
    run_prompt([300, 129, 1], [0, 500, 1100], heads, types, seed=3, pad=16)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("max_len", [0, 1, 2100, 1 << 30])
def test_few_rows_behind_a_long_cache(types, max_len):
    run_prompt([3, 8, 1], [2000, 1023, 17], (8, 2, 128), types, seed=4, max_len=max_len)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_more_sequences_than_a_wave(types):
    rng = random.Random(1)
    run_prompt([rng.choice([0, 1, 1, 2, 5]) for _ in range(150)], [rng.choice([0, 0, 3, 40]) for _ in range(150)], (4, 2, 64), types)


@pytest.mark.parametrize("heads,rows,cached", [((128, 8, 64), [700, 1, 450], [0, 70, 333]), ((64, 8, 128), [1, 2300, 33], [5, 0, 1000]),
                                               ((96, 16, 128), [1500, 15], [7, 0])], ids=str)
def test_batches_of_many_rows(heads, rows, cached):
    """Past the size from which a wave takes 64 queries; rows at the tiles' edges and a few others are compared."""
    from tests.seqcache import attend, check, filled, i32
    hq, hkv, dh = heads
    assert sum(rows) * hq >= 512 * 256
    lens = [r + c for r, c in zip(rows, cached)]
    cache, kv = filled(lens, hkv, dh, torch.bfloat16, 21)
    cu = [0]
    for r in rows:
        cu.append(cu[-1] + r)
    q = (1.5 * torch.randn(cu[-1], hq, dh, generator=torch.Generator().manual_seed(22))).bfloat16()
    out = cache.prompt_attention(0, q.cuda(), i32(list(range(len(rows)))), i32(cu)).cpu()
    assert torch.isfinite(out).all()
    G = hq // hkv
    for i, n in enumerate(rows):
        rpt = 256 // G
        pick = sorted({r for r in (0, 1, rpt - 1, rpt, 3 * rpt - 1, n // 2, n - 2, n - 1) if 0 <= r < n})
        want, mag = attend(q[cu[i]:cu[i + 1]][pick], kv[i][0, 0], kv[i][0, 1], [cached[i] + r + 1 for r in pick])
        check(out[cu[i]:cu[i + 1]][pick], want, mag, ("bf16", i))


def run_prefix(groups, prefix, lens, heads, types, seed=0, max_len=0, pad=0, use_groups=True):
    """Groups of rows that agree in their first prefix keys, in pages of their own."""
    from tests.seqcache import agree, attend, check, filled, i32
    hq, hkv, dh = heads
    n = len(lens)
    cache, kv = filled(lens, hkv, dh, dt(types[1]), seed)
    cu = [0]
    for r in groups:
        cu.append(cu[-1] + r)
    for j in range(len(groups)):
        for i in range(cu[j] + 1, cu[j + 1]):
            agree(cache, cu[j], i, min(prefix[j], lens[cu[j]], lens[i]))
    g = torch.Generator().manual_seed(seed + 1)
    wide = (1.5 * torch.randn(n, hq * dh + pad, generator=g)).to(dt(types[0])).cuda()
    q = wide[:, :hq * dh].unflatten(1, (hq, dh))
    out = torch.full((n, hq * dh + pad), 7.0, dtype=dt(types[0]), device="cuda")
    print(f"[prefix {types} {heads} groups {groups} prefix {prefix} lens {lens}]", flush=True)
    extra = (i32(cu), i32(prefix)) if use_groups else ()
    cache.prefix_attention(0, q, i32(list(range(n))), *extra, out=out[:, :hq * dh].unflatten(1, (hq, dh)), max_len=max_len)
    torch.cuda.synchronize()
    for j in range(len(groups)):
        for i in range(cu[j], cu[j + 1]):
            p = min(prefix[j], lens[cu[j]])
            m = min(p, lens[i])
            x = torch.cat([kv[cu[j]][0, :, :, :m], kv[i][0, :, :, m:]], 2)
            want, mag = attend(q[i:i + 1], x[0], x[1], [lens[i]])
            check(out[i:i + 1, :hq * dh].unflatten(1, (hq, dh)), want, mag, (types[0], "row", i))
    assert (out[:, hq * dh:] == 7.0).all()


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_shared_prefixes(heads, types):
    run_prefix([3, 1, 0, 5, 1], [100, 0, 64, 33, 1], [130, 100, 101, 1, 200, 33, 34, 40, 16, 5], heads, types, pad=8)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_rows_without_keys_and_prefixes_of_any_length(types):
    """Sequences without keys, rows shorter than the prefix of their group, prefixes past the first row's keys."""
    run_prefix([4, 2, 2], [50, 16, 1000], [70, 0, 20, 50, 0, 9, 30, 45], (8, 2, 128), types, seed=2)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("max_len", [0, 5, 3000])
def test_long_prefix(types, max_len):
    run_prefix([21, 40], [2500, 777], [2500 + 7 * i for i in range(21)] + [777 + 13 * i for i in range(40)], (8, 2, 128), types,
               seed=5, max_len=max_len)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)], ids=str)
def test_short_shared_prefixes(heads, types):
    for max_len in (100, 512):
        run_prefix([3, 1, 2], [37, 9, 64], [40, 99, 37, 20, 70, 65], heads, types, seed=9, max_len=max_len)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_no_groups(types):
    run_prefix([1] * 4, [0] * 4, [1, 17, 900, 64], (8, 2, 128), types, seed=6, use_groups=False)


def test_many_rows():
    rng = random.Random(3)
    groups = [rng.choice([0, 1, 1, 7, 40]) for _ in range(70)]
    prefix = [rng.choice([0, 16, 30]) for _ in groups]
    lens = [p + rng.randint(0, 9) for r, p in zip(groups, prefix) for _ in range(r)]
    run_prefix(groups, prefix, lens, (4, 2, 64), ("bf16", "bf16"), seed=7)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_values_that_are_not_finite_stay_with_the_rows_that_attend_them(types):
    """An infinity or NaN in a key or value reaches the rows at and behind its position, as in plain arithmetic, and
    no row before; what stale memory holds reaches none."""
    from tests.seqcache import filled, i32
    n, heads, dh = 90, (8, 2), 128
    for where, what in (("k", float("nan")), ("v", float("inf")), ("v", float("nan")), ("k", float("-inf"))):
        cache, kv = filled([n], heads[1], dh, dt(types[1]), 11)
        page = int(cache.page_table[0, 40 // 16])
        cache.kv[0, page, 0 if where == "k" else 1, 1, 40 % 16, 5] = what
        q = torch.randn(n, heads[0], dh, generator=torch.Generator().manual_seed(1)).to(dt(types[0])).cuda()
        out = cache.prompt_attention(0, q, i32([0]), i32([0, n])).double().cpu()
        x = kv[0][0].double()
        x[0 if where == "k" else 1, 1, 40, 5] = what
        s = torch.einsum("nhd,hkd->nhk", q.double().cpu(), x[0].repeat_interleave(4, 0)) / dh ** 0.5
        late = torch.arange(n)[None, :] > torch.arange(n)[:, None]
        p = torch.softmax(s.masked_fill(late[:, None], float("-inf")), -1)
        # a masked key has no part in the sum, whatever its value
        want = torch.stack([torch.einsum("hk,hkd->hd", p[i, :, :i + 1], x[1, :, :i + 1].repeat_interleave(4, 0)) for i in range(n)])
        assert torch.equal(torch.isnan(out), torch.isnan(want)), (where, what)
        assert torch.equal(torch.isinf(out), torch.isinf(want)), (where, what)
        fin = torch.isfinite(want)
        assert ((out - want)[fin].abs() <= (2 ** -6 if types[0] == "bf16" else 1e-4) * 4.0).all()
        one = cache.prefix_attention(0, q[-1:].contiguous(), i32([0]), i32([0, 1]), i32([50])).double().cpu()
        assert torch.equal(torch.isfinite(one), torch.isfinite(want[-1:])), (where, what)


def test_lengths_and_pages_out_of_range_read_nothing_outside():
    """Lengths past the table, ids that are no pages, sequences that do not exist: bounded, and other rows are right."""
    from tests.seqcache import attend, check, filled, i32
    cache, kv = filled([40, 33, 20], 2, 64, torch.bfloat16, 3, stale=0.0)
    cache.page_table[0, 1] = 1 << 30
    cache.page_table[0, 2] = -7
    cache.lens[0] = 1 << 30
    cache.lens[2] = -5
    q = torch.randn(9, 4, 64, device="cuda").bfloat16()
    out = torch.full_like(q, 7.0)
    cache.prompt_attention(0, q, i32([0, 1, 9, 2, -1]), i32([0, 2, 5, 6, 8, 9]), out=out)
    want, mag = attend(q[2:5], kv[1][0, 0], kv[1][0, 1], [31, 32, 33])
    check(out[2:5], want, mag, ("bf16",))
    assert (out[5] == 7.0).all() and (out[8] == 7.0).all() and (out[6:8] == 0).all()
    out = cache.prefix_attention(0, q[:3], i32([0, 1, 2]), i32([0, 3]), i32([1 << 30]))
    torch.cuda.synchronize()
    assert (out[2] == 0).all()


@pytest.mark.parametrize("kind", ["prompt", "prefix"])
def test_captured_calls_follow_the_lengths(kind):
    """A captured call on lengths that change between its replays, beside eager calls."""
    from tests.seqcache import i32, filled
    cache, kv = filled([200, 90], 2, 128, torch.bfloat16, 8)
    q = torch.randn(2, 8, 128, device="cuda").bfloat16()
    seqs, cu = i32([0, 1]), i32([0, 1, 2])

    def call():
        if kind == "prompt":
            return cache.prompt_attention(0, q, seqs, cu)
        return cache.prefix_attention(0, q, seqs, i32_cu, pre)

    i32_cu, pre = i32([0, 1, 2]), i32([64, 16])
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call()
    for lens in ([200, 90], [3, 64], [0, 17], [161, 1], [200, 90]):
        cache.lens.copy_(i32(lens))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, call()), lens
        torch.cuda.synchronize()
