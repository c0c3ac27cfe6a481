"""Attention under a rule over a cache of several sequences, against 64 bits: packed rows, and decode rows of groups that share a
prefix, with every part of a rule alone and all of them at once."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]
HEADS = [(8, 2, 128), (4, 4, 64), (6, 2, 64), (16, 1, 128), (5, 1, 128)]
PARTS = ["", "cap", "slopes", "window", "docs", "open", "cap slopes", "window open", "cap slopes window docs open"]


def dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def slopes_of(hq):
    return [2.0 ** (-6.0 * (h + 1) / hq) for h in range(hq)]


def make(parts, rng, rows, cached, hq, window=None):
    """The rule's plain values: cap, slopes, window, and for each row its first key, for each sequence its open keys."""
    from tests.ruled import FAR
    cap = 7.0 if "cap" in parts else 0.0
    slopes = slopes_of(hq) if "slopes" in parts else None
    window = (window or rng.choice([1, 16, 30, 70])) if "window" in parts else 0
    first = None
    if "docs" in parts:
        first = []
        for r, c in zip(rows, cached):
            at = 0
            for i in range(r):
                if rng.random() < 0.06:
                    at = c + i
                first.append(FAR if rng.random() < 0.06 else 0 if rng.random() < 0.06 else at)
    opened = [rng.choice([0, 1, 16, r + c, (r + c) // 2, 5]) for r, c in zip(rows, cached)] if "open" in parts else None
    return cap, slopes, window, first, opened


def rule_of(cap, slopes, window, first, opened, tail=0):
    from paper_2605_30852_amd.cache import AttentionRule
    from tests.seqcache import i32
    return AttentionRule(cap=cap, slopes=torch.tensor(slopes, device="cuda") if slopes is not None else None, window=window,
                         first=i32(first + [0] * tail) if first is not None else None, open_lens=i32(opened) if opened is not None else None)


def run_prompt(rows, cached, heads, types, parts, seed=0, tail=0, max_len=0, pad=0, window=None, made=None, some=None):
    from tests.ruled import attend, check
    from tests.seqcache import filled, i32
    hq, hkv, dh = heads
    rng = random.Random(seed)
    n = len(rows)
    slots = rng.sample(range(n), n)
    lens = [0] * n
    for i, s in enumerate(slots):
        lens[s] = rows[i] + cached[i]
    cache, kv = filled(lens, hkv, dh, dt(types[1]), seed)
    cap, slopes, window, first, opened = made or make(parts, rng, rows, cached, hq, window)
    cu = [0]
    for r in rows:
        cu.append(cu[-1] + r)
    total = cu[-1] + tail
    g = torch.Generator().manual_seed(seed + 1)
    wide = (1.5 * torch.randn(total, hq * dh + pad, generator=g)).to(dt(types[0])).cuda()
    q = wide[:, :hq * dh].unflatten(1, (hq, dh))
    out = torch.full((total, hq * dh + pad), 7.0, dtype=dt(types[0]), device="cuda")
    print(f"[ruled prompt {types} {heads} rows {rows} cached {cached} {parts}]", flush=True)
    cache.prompt_attention(0, q, i32(slots), i32(cu), out=out[:, :hq * dh].unflatten(1, (hq, dh)), max_len=max_len,
                           rule=rule_of(cap, slopes, window, first, opened, tail))
    torch.cuda.synchronize()
    for i, s in enumerate(slots):
        pick = [r for r in range(rows[i]) if some is None or r % some == 0 or r == rows[i] - 1]
        if not pick:
            continue
        at = [cu[i] + r for r in pick]
        sees = [(cached[i] + r, first[cu[i] + r] if first else 0, opened[i] if opened else 0) for r in pick]
        want, mag = attend(q[at], kv[s][0, 0], kv[s][0, 1], sees, cap, slopes, window)
        check(out[at, :hq * dh].unflatten(1, (hq, dh)), want, mag, (types[0], "sequence", i))
    assert (out[cu[-1]:] == 7.0).all() and (out[:, hq * dh:] == 7.0).all()


@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_each_part(types, parts):
    """Pieces of wide tiles, and (max_len) one launch of few queries."""
    for max_len in (0, 200):
        run_prompt([1, 17, 0, 64, 33], [0, 15, 5, 0, 110], (8, 2, 128), types, parts, tail=3, max_len=max_len)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("heads", HEADS[1:], ids=str)
def test_heads(heads, types):
    for max_len in (0, 200):
        run_prompt([1, 2, 17, 0, 64, 65], [0, 15, 100, 5, 0, 1], heads, types, PARTS[-1], seed=max_len, max_len=max_len, pad=16)


@pytest.mark.parametrize("parts", ["cap", "slopes", "window open", "docs open", "cap slopes window docs open"])
@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_long_prompts(types, parts):
    run_prompt([300, 129, 1], [0, 500, 1100], (8, 2, 128), types, parts, seed=3, window=150, some=7)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("parts", ["cap slopes", "window open", "docs"])
def test_few_rows_behind_a_long_cache(types, parts):
    """Pieces of few queries whose keys are split, and a gap inside them."""
    run_prompt([3, 8, 1, 2], [2000, 1023, 17, 2600], (8, 2, 128), types, parts, seed=4, window=900)
    run_prompt([3, 8, 1, 2], [2000, 1023, 17, 2600], (6, 2, 64), types, parts, seed=5, window=40)


def test_rows_that_see_nothing():
    """No key at all: zeros; one key; open keys alone."""
    from tests.ruled import FAR
    n = [20, 40]
    for types in TYPES:
        first = [FAR if i % 3 else i - 20 if i >= 20 else i for i in range(60)]
        for max_len in (0, 64):
            run_prompt(n, [0, 0], (8, 2, 128), types, "nothing", made=(0.0, None, 0, first, None), max_len=max_len)
            run_prompt(n, [0, 0], (8, 2, 128), types, "nothing", made=(5.0, slopes_of(8), 0, [FAR] * 60, [0, 3]), max_len=max_len)
            run_prompt(n, [0, 0], (8, 2, 128), types, "one", made=(0.0, None, 1, None, None), max_len=max_len)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_far_keys_alone(types):
    """Rows that see keys some thousands behind them, under steep slopes: the distance counts from the nearest that they see."""
    from tests.ruled import FAR
    steep = [5.0, 0.5, 0.05, 30.0]
    run_prompt([40], [9000], (4, 1, 128), types, "far", made=(0.0, steep, 0, [FAR] * 40, [37]), some=5)
    run_prompt([40], [9000], (4, 1, 128), types, "far", made=(9.0, steep, 3, None, [37]), some=5)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), "lowest"])
def test_unseen_keys_may_hold_anything(types, bad):
    """Keys and values outside every row's window and document, and behind a row, at the ends of the type's range."""
    from tests.ruled import attend, check
    from tests.seqcache import filled, i32
    hq, hkv, dh = 8, 2, 128
    if bad == "lowest":
        bad = torch.finfo(dt(types[1])).min
    for max_len in (0, 400):
        cache, kv = filled([300], hkv, dh, dt(types[1]), 8)
        j = torch.arange(300, device="cuda")
        page = cache.page_table[0].long()[j // 16]
        for unseen in (slice(3, 150), slice(290, 300)):  # the row of key 289 and those before it
            cache.kv[0, page[unseen], :, :, j[unseen] % 16] = bad
        q = (1.5 * torch.randn(120, hq, dh, generator=torch.Generator().manual_seed(1))).to(dt(types[0])).cuda()
        rule = rule_of(7.0, slopes_of(hq), 31, None, [3])
        cache.lens[0] = 300
        out = cache.prompt_attention(0, q, i32([0]), i32([0, 120]), max_len=max_len, rule=rule)
        rows = list(range(109))
        want, mag = attend(q[:109], kv[0][0, 0], kv[0][0, 1], [(180 + r, 0, 3) for r in rows], 7.0, slopes_of(hq), 31)
        check(out[:109], want, mag, (types[0], bad))


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_scores_at_the_ends_of_a_cap(types):
    """Scores far above a cap are the cap, also infinite ones; small caps and large ones."""
    from tests.ruled import attend, check
    from tests.seqcache import filled, i32
    hq, hkv, dh = 4, 2, 64
    for cap in (2.0 ** -20, 0.01, 1.0, 50.0, 1000.0, 2.0 ** 20):
        cache, kv = filled([70], hkv, dh, dt(types[1]), 9)
        q = (1.5 * torch.randn(70, hq, dh, generator=torch.Generator().manual_seed(2))).to(dt(types[0])).cuda()
        q[::5] *= 40.0
        q[1::5] *= 1e-3
        out = cache.prompt_attention(0, q, i32([0]), i32([0, 70]), rule=rule_of(cap, None, 0, None, None))
        want, mag = attend(q, kv[0][0, 0], kv[0][0, 1], [(r, 0, 0) for r in range(70)], cap)
        keep = [r for r in range(70) if r % 5 or cap <= 50.0]  # forty times the scores, uncapped: forty times their error
        check(out[keep], want[keep], mag[keep], (types[0], cap))
    cache, kv = filled([70], hkv, dh, dt(types[1]), 10)
    q = torch.zeros(70, hq, dh, dtype=dt(types[0]), device="cuda")
    q[..., 0] = 1.0
    k = kv[0][0, 0].clone()
    k[:, ::3, 0] = float("inf")
    k[:, 1::3, 0] = float("-inf")
    j = torch.arange(70, device="cuda")
    page = cache.page_table[0].long()[j // 16]
    cache.kv[0, page, 0, :, j % 16] = k.transpose(0, 1).cuda()
    out = cache.prompt_attention(0, q, i32([0]), i32([0, 70]), rule=rule_of(3.0, None, 0, None, None))
    want, mag = attend(q.double().where(q != 0, torch.tensor(1e-200, dtype=torch.float64, device="cuda")),
                       torch.nan_to_num(k.double(), posinf=1e300, neginf=-1e300), kv[0][0, 1], [(r, 0, 0) for r in range(70)], 3.0)
    check(out, want, mag, (types[0], "infinite"))


def run_prefix(groups, prefix, lens, heads, types, parts, seed=0, max_len=0, window=None, use_groups=True):
    from tests.ruled import attend, check
    from tests.seqcache import agree, filled, i32
    hq, hkv, dh = heads
    rng = random.Random(seed)
    n = len(lens)
    cache, kv = filled(lens, hkv, dh, dt(types[1]), seed)
    cu = [0]
    for r in groups:
        cu.append(cu[-1] + r)
    for j in range(len(groups)):
        for i in range(cu[j] + 1, cu[j + 1]):
            agree(cache, cu[j], i, min(prefix[j], lens[cu[j]], lens[i]))
    cap, slopes, window, first, opened = make(parts, rng, [1] * n, [max(0, x - 1) for x in lens], hq, window)
    q = (1.5 * torch.randn(n, hq, dh, generator=torch.Generator().manual_seed(seed + 1))).to(dt(types[0])).cuda()
    print(f"[ruled prefix {types} {heads} groups {groups} prefix {prefix} {parts}]", flush=True)
    extra = (i32(cu), i32(prefix)) if use_groups else ()
    out = cache.prefix_attention(0, q, i32(list(range(n))), *extra, max_len=max_len, rule=rule_of(cap, slopes, window, first, opened))
    torch.cuda.synchronize()
    for j in range(len(groups)):
        for i in range(cu[j], cu[j + 1]):
            m = min(prefix[j], lens[cu[j]], lens[i])
            x = torch.cat([kv[cu[j]][0, :, :, :m], kv[i][0, :, :, m:]], 2)
            sees = [(lens[i] - 1, first[i] if first else 0, min(opened[i], lens[i]) if opened else 0)]
            want, mag = attend(q[i:i + 1], x[0], x[1], sees, cap, slopes, window)
            check(out[i:i + 1], want, mag, (types[0], "row", i))


@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_decode_rows(types, parts):
    for max_len in (0, 512):
        run_prefix([1] * 7, [0] * 7, [1, 0, 16, 17, 300, 511, 90], (8, 2, 128), types, parts, max_len=max_len, use_groups=False)
    run_prefix([1] * 4, [0] * 4, [2100, 1, 700, 3500], (5, 1, 128), types, parts, use_groups=False, window=600)


@pytest.mark.parametrize("parts", PARTS[1:])
@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_groups(types, parts):
    rng = random.Random(7)
    groups, prefix = [3, 1, 20, 2], [200, 40, 333, 0]
    lens = [p + rng.choice([0, 1, 3, 90]) for g, p in zip(groups, prefix) for _ in range(g)]
    lens[1] -= 30  # shorter than its group's prefix
    for max_len in (0, 512):
        run_prefix(groups, prefix, lens, (8, 2, 128), types, parts, seed=2, max_len=max_len, window=60)
    run_prefix(groups, prefix, lens, (6, 2, 64), types, parts, seed=3, window=120)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_long_prefixes(types):
    lens = [2300 + 7 * i for i in range(12)]
    for parts, window in (("cap slopes", None), ("window open", 200), ("window", 5), ("cap slopes window docs open", 2290)):
        run_prefix([12], [2300], lens, (8, 2, 128), types, parts, seed=4, window=window)


def test_a_rule_of_nothing_is_no_rule():
    from paper_2605_30852_amd.cache import AttentionRule
    from tests.seqcache import filled, i32
    for types in TYPES:
        cache, _ = filled([400, 90], 2, 128, dt(types[1]), 4)
        q = torch.randn(190, 8, 128, generator=torch.Generator().manual_seed(3)).to(dt(types[0])).cuda()
        for max_len in (0, 400):
            a = cache.prompt_attention(0, q, i32([0, 1]), i32([0, 100, 190]), max_len=max_len)
            b = cache.prompt_attention(0, q, i32([0, 1]), i32([0, 100, 190]), max_len=max_len, rule=AttentionRule())
            assert torch.equal(a, b)


def test_rules_of_other_sizes_are_refused():
    from paper_2605_30852_amd.cache import AttentionRule
    from tests.seqcache import filled, i32
    cache, _ = filled([40, 9], 2, 64, torch.float32, 4)
    q = torch.randn(5, 4, 64, device="cuda")
    for rule in (AttentionRule(slopes=torch.ones(2, device="cuda")), AttentionRule(first=i32([0] * 4)), AttentionRule(open_lens=i32([0]))):
        with pytest.raises(ValueError):
            cache.prompt_attention(0, q, i32([0, 1]), i32([0, 3, 5]), rule=rule)
        with pytest.raises(ValueError):
            cache.prefix_attention(0, q[:2], i32([0, 1]), rule=AttentionRule(first=i32([0] * 3)))


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_in_a_graph(types):
    """Captured calls follow the lengths, the documents and the open keys on replay, with eager calls in between."""
    from tests.seqcache import filled, i32
    cache, _ = filled([700, 300], 2, 128, dt(types[1]), 6)
    g = torch.Generator().manual_seed(5)
    q = torch.randn(60, 8, 128, generator=g).to(dt(types[0])).cuda()
    first, opened, seqs, cu = i32([0] * 60), i32([0, 9]), i32([0, 1]), i32([0, 40, 60])
    from paper_2605_30852_amd.cache import AttentionRule
    rule = AttentionRule(cap=6.0, slopes=torch.tensor(slopes_of(8), device="cuda"), window=200, first=first, open_lens=opened)
    rows = AttentionRule(cap=6.0, window=90, open_lens=opened)

    def both():
        return (cache.prompt_attention(0, q, seqs, cu, rule=rule), cache.prefix_attention(0, q[:2], seqs, rule=rows),
                cache.prompt_attention(0, q, seqs, cu, max_len=256, rule=rule))

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for k in range(4):
        first.copy_(i32([(37 * i * k) % 650 for i in range(60)]))
        opened.copy_(i32([5 * k, 100 * k]))
        cache.lens.copy_(i32([700 - 60 * k, 256 + 3 * k]))
        want = [x.clone() for x in both()]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), k


def test_two_streams_at_once():
    """Calls on two streams have workspaces of their own."""
    from tests.seqcache import filled, i32
    cache, _ = filled([900, 1100], 2, 128, torch.bfloat16, 6)
    q = torch.randn(200, 8, 128, generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    rule = rule_of(6.0, slopes_of(8), 300, None, [7, 9])
    args = (0, q, i32([0, 1]), i32([0, 120, 200]))
    want = cache.prompt_attention(*args, rule=rule)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(cache.prompt_attention(*args, rule=rule))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_a_layer_of_another_decoder(types):
    """A run of the operators as they are used: pages, a scaled table, normed heads, prompts, then steps of samples that share a prompt."""
    from paper_2605_30852_amd.cache import AttentionRule, HeadRule, PagedCache
    from paper_2605_30852_amd.rope import RopeScaling, rope_frequencies, rope_table
    from tests.ruled import attend, check, turned
    from tests.seqcache import i32
    hq, hkv, dh, rot = 8, 2, 128, 64
    cache = PagedCache.empty(1, 60, hkv, dh, 4, 12, dtype=dt(types[1]))
    cos, sin = rope_table(rope_frequencies(rot, 10000.0, RopeScaling("parts", 4.0, 64, 1.0, 8.0)), 16 * cache.max_pages, amplitude=1.1)
    g = torch.Generator().manual_seed(11)
    gains = [(1 + 0.2 * torch.randn(dh, generator=g)).cuda() for _ in range(2)]
    heads = HeadRule(q_gain=gains[0], k_gain=gains[1], interleaved=True)
    slopes = slopes_of(hq)
    rule = AttentionRule(cap=20.0, slopes=torch.tensor(slopes, device="cuda"), window=50)
    keys = {s: [] for s in range(4)}  # what the cache holds, as it was rounded

    def put(seqs, rows):
        cu = [0]
        for r in rows:
            cu.append(cu[-1] + r)
        x = torch.randn(cu[-1], hq + 2 * hkv, dh, generator=g).to(dt(types[0])).cuda()
        old = cache.lens.tolist()
        assert cache.reserve(i32(seqs), i32(rows)).item() == 0
        q = cache.append_heads(0, x[:, hq:hq + hkv], x[:, hq + hkv:], i32(seqs), i32(cu), heads, q=x[:, :hq], rope=(cos, sin))
        for i, s in enumerate(seqs):
            pos = torch.arange(old[s], old[s] + rows[i])
            k, _ = turned(x[cu[i]:cu[i + 1], hq:hq + hkv].cpu(), pos, gains[1].cpu(), 1e-6, (cos.cpu(), sin.cpu()), True)
            page = cache.page_table[s].cpu().long()[pos // 16]
            now = cache.kv[0].cpu()[page, 0, :, pos % 16].double()
            assert ((now - k).abs() <= (2 ** -8 if types[1] == "bf16" else 2 ** -18) * (k.abs() + 1)).all()
        return q, cu

    def held(s):
        n = int(cache.lens[s])
        j = torch.arange(n, device="cuda")
        x = cache.kv[0, cache.page_table[s].long()[j // 16], :, :, j % 16]
        return x[:, 0].transpose(0, 1), x[:, 1].transpose(0, 1), n

    q, cu = put([0, 1], [70, 33])
    out = cache.prompt_attention(0, q, i32([0, 1]), i32(cu), rule=rule)
    for i, s in enumerate([0, 1]):
        k, v, n = held(s)
        want, mag = attend(q[cu[i]:cu[i + 1]], k, v, [(r, 0, 0) for r in range(n)], 20.0, slopes, 50)
        check(out[cu[i]:cu[i + 1]], want, mag, (types[0], "prompt", s))
    assert cache.fork(i32([0, 0]), i32([2, 3]), i32([70, 70])).item() == 0
    for step in range(3):
        order = [0, 2, 3, 1]
        q, _ = put(order, [1] * 4)
        out = cache.prefix_attention(0, q, i32(order), i32([0, 3, 4]), i32([70, 0]), rule=rule)
        for i, s in enumerate(order):
            k, v, n = held(s)
            want, mag = attend(q[i:i + 1], k, v, [(n - 1, 0, 0)], 20.0, slopes, 50)
            check(out[i:i + 1], want, mag, (types[0], "step", step, s))


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("cap", [0.0, 500.0])
def test_scores_far_below_zero(types, cap):
    """Every score of a row some hundreds below 0, and keys that the distance lowers as much: one piece, split pieces, a shared prefix."""
    from tests.ruled import attend
    from tests.seqcache import filled, i32
    hq, hkv, dh = 4, 1, 128
    steep = [20.0, 2.0, 0.02, 0.0]
    for n, new in ((300, 300), (2500, 40)):
        cache, kv = filled([n], hkv, dh, dt(types[1]), 12)
        k = kv[0][0, 0].clone()
        k[..., 0] = -300.0
        j = torch.arange(n, device="cuda")
        page = cache.page_table[0].long()[j // 16]
        cache.kv[0, page, 0, :, j % 16] = k.transpose(0, 1).cuda()
        q = torch.randn(new, hq, dh, generator=torch.Generator().manual_seed(4)).to(dt(types[0])).cuda()
        q[..., 0] = 12.0
        rule = rule_of(cap, steep, 0, None, None)
        out = cache.prompt_attention(0, q, i32([0]), i32([0, new]), rule=rule)
        rows = [r for r in range(new) if r % 9 == 0 or r > new - 3]
        want, mag = attend(q[rows], k, kv[0][0, 1], [(n - new + r, 0, 0) for r in rows], cap, steep)
        # a score of 300 beside products of 3600 / sqrt(128): fp32 holds it to some 128 roundings of 2^-24 of 318, a few 1e-5 each way; three
        # planes of a query likewise; with a cap of 500 the tanh of it, off by 2^-22 of 280
        bound = (2e-3 + (2 ** -7 if types[0] == "bf16" else 0.0)) * (mag + want.abs())
        assert torch.isfinite(out).all() and ((out[rows].double().cpu() - want).abs() <= bound).all(), (n, cap)
    cache, kv = filled([2400, 2400], hkv, dh, dt(types[1]), 13)
    from tests.seqcache import agree
    for s in range(2):
        j = torch.arange(2400, device="cuda")
        page = cache.page_table[s].long()[j // 16]
        cache.kv[0, page, 0, :, j % 16, 0] = -300.0
    agree(cache, 0, 1, 2300)
    q = torch.randn(2, hq, dh, generator=torch.Generator().manual_seed(4)).to(dt(types[0])).cuda()
    q[..., 0] = 12.0
    out = cache.prefix_attention(0, q, i32([0, 1]), i32([0, 2]), i32([2300]), rule=rule_of(cap, steep, 0, None, None))
    for s in range(2):
        j = torch.arange(2400, device="cuda")
        x = cache.kv[0, cache.page_table[s].long()[j // 16], :, :, j % 16]
        want, mag = attend(q[s:s + 1], x[:, 0].transpose(0, 1), x[:, 1].transpose(0, 1), [(2399, 0, 0)], cap, steep)
        bound = (2e-3 + (2 ** -7 if types[0] == "bf16" else 0.0)) * (mag + want.abs())
        assert ((out[s:s + 1].double().cpu() - want).abs() <= bound).all(), (s, cap)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_small_values_under_a_cap(types):
    """Every score at the lower end of the cap, and values of 2^-40: nothing of them is lost."""
    from tests.ruled import attend, check
    from tests.seqcache import filled, i32
    hq, hkv, dh = 4, 2, 128
    cache, kv = filled([200], hkv, dh, dt(types[1]), 14)
    k, v = kv[0][0, 0].clone(), kv[0][0, 1] * 2.0 ** -40
    k[..., 0] = -3000.0
    j = torch.arange(200, device="cuda")
    page = cache.page_table[0].long()[j // 16]
    cache.kv[0, page, 0, :, j % 16] = k.transpose(0, 1).cuda()
    cache.kv[0, page, 1, :, j % 16] = v.transpose(0, 1).cuda()
    q = torch.randn(200, hq, dh, generator=torch.Generator().manual_seed(4)).to(dt(types[0])).cuda()
    q[..., 0] = 12.0
    for slopes in (None, slopes_of(hq)):
        out = cache.prompt_attention(0, q, i32([0]), i32([0, 200]), rule=rule_of(55.0, slopes, 0, None, None))
        want, mag = attend(q, k, v, [(r, 0, 0) for r in range(200)], 55.0, slopes)
        check(out, want, mag, (types[0], slopes))


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_open_lengths_and_first_keys_out_of_range(types):
    """A sequence's open keys are at most its own, none below 0; first keys below 0 are the first."""
    from tests.ruled import attend, check
    from tests.seqcache import filled, i32
    hq, hkv, dh = 8, 2, 64
    cache, kv = filled([90, 40], hkv, dh, dt(types[1]), 15)
    q = (1.5 * torch.randn(70, hq, dh, generator=torch.Generator().manual_seed(6))).to(dt(types[0])).cuda()
    for opened in ([1 << 30, -7], [-1 << 31, (1 << 31) - 1]):
        first = [-5 - i for i in range(70)]
        for max_len in (0, 90):
            out = cache.prompt_attention(0, q, i32([0, 1]), i32([0, 30, 70]), max_len=max_len, rule=rule_of(7.0, None, 9, first, opened))
            for i, (a, b, n) in enumerate(((0, 30, 90), (30, 70, 40))):
                want, mag = attend(q[a:b], kv[i][0, 0], kv[i][0, 1], [(n - (b - r), 0, min(max(opened[i], 0), n)) for r in range(a, b)], 7.0, None, 9)
                check(out[a:b], want, mag, (types[0], opened, i))


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_many_decode_rows_under_a_window(types):
    """As many rows as fill the GPU go without a plan, whatever their lengths and open keys."""
    from tests.ruled import attend, check
    from tests.seqcache import filled, i32
    hq, hkv, dh = 8, 8, 64
    rng = random.Random(8)
    lens = [rng.choice([0, 1, 15, 700, 701, 1500, rng.randint(1, 1900)]) for _ in range(66)]
    opened = [rng.choice([0, 1, 4, 33, n]) for n in lens]
    cache, kv = filled(lens, hkv, dh, dt(types[1]), 16)
    q = (1.5 * torch.randn(66, hq, dh, generator=torch.Generator().manual_seed(6))).to(dt(types[0])).cuda()
    slopes = slopes_of(hq)
    for max_len in (0, 1900):
        seqs = list(range(66))
        seqs[5] = 66  # none
        out = torch.full_like(q, 7.0)
        cache.prefix_attention(0, q, i32(seqs), out=out, max_len=max_len, rule=rule_of(7.0, slopes, 700, None, opened))
        for s in range(66):
            if s == 5:
                assert (out[s] == 7.0).all()
                continue
            want, mag = attend(q[s:s + 1], kv[s][0, 0], kv[s][0, 1], [(lens[s] - 1, 0, opened[s])], 7.0, slopes, 700)
            check(out[s:s + 1], want, mag, (types[0], s))


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("cap", [0.0, 7.0])
def test_scores_that_rise_with_the_distance(types, cap):
    """Slopes below 0: the farthest keys count most."""
    from tests.ruled import attend, check
    from tests.seqcache import filled, i32
    hq, hkv, dh = 4, 2, 128
    cache, kv = filled([900], hkv, dh, dt(types[1]), 17)
    q = (1.5 * torch.randn(200, hq, dh, generator=torch.Generator().manual_seed(6))).to(dt(types[0])).cuda()
    slopes = [-0.01, -0.002, 0.0, -0.02]
    out = cache.prompt_attention(0, q, i32([0]), i32([0, 200]), rule=rule_of(cap, slopes, 0, None, None))
    rows = list(range(0, 200, 7))
    want, mag = attend(q[rows], kv[0][0, 0], kv[0][0, 1], [(700 + r, 0, 0) for r in rows], cap, slopes)
    check(out[rows], want, mag, (types[0], cap))


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_a_large_pool(types):
    """Pages whose bytes lie past 2^32 of the pool."""
    from paper_2605_30852_amd.cache import AttentionRule, PagedCache
    from tests.ruled import attend, check
    from tests.seqcache import i32
    hkv, dh, item = 8, 128, 2 if types[1] == "bf16" else 4
    page = 2 * hkv * 16 * dh * item
    num = (1 << 32) // page + 40
    cache = PagedCache.empty(1, num, hkv, dh, 1, 32, dtype=dt(types[1]))
    ids = [num - 1 - 2 * i for i in range(13)]
    cache.page_table[0, :13] = i32(ids)
    cache.lens[0] = 200
    g = torch.Generator().manual_seed(3)
    x = torch.randn(13, 2, hkv, 16, dh, generator=g).to(dt(types[1]))
    cache.kv[0, ids] = x.cuda()
    k, v = (x[:, i].transpose(0, 1).flatten(1, 2)[:, :200] for i in range(2))
    q = (1.5 * torch.randn(40, 16, dh, generator=g)).to(dt(types[0])).cuda()
    out = cache.prompt_attention(0, q, i32([0]), i32([0, 40]), rule=AttentionRule(cap=7.0, window=90))
    want, mag = attend(q[::5], k, v, [(160 + r, 0, 0) for r in range(0, 40, 5)], 7.0, None, 90)
    check(out[::5], want, mag, (types[0],))
