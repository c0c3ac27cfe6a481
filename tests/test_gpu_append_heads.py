"""Normed and rotated heads into the pages of several sequences, against 64 bits."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32"), ("bf16", "f32")]


def dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def within(got, want, mag, name, what):
    """A norm is off by its sum of squares, 16 terms of a lane and 3 joins: 19 roundings of 2^-24, half of them in its root, and four
    more; a rotation by three roundings of its two terms; and the result by half a step, 2^-8 or 2^-24 of it."""
    bound = 17 * 2 ** -24 * mag + (2 ** -8 if name == "bf16" else 2 ** -24) * want.abs() + 1e-37
    assert ((got.double().cpu() - want).abs() <= bound).all(), what


def case(rows, cached, heads, types, rot, interleaved, gains, seed=0, tail=0, scale=1.7, in_place=False, with_q=True, packed=True):
    from paper_2605_30852_amd.cache import HeadRule
    from tests.ruled import turned
    from tests.seqcache import PAGE, filled, i32
    hq, hkv, dh = heads
    rng = random.Random(seed)
    n = len(rows)
    slots = rng.sample(range(n), n)
    lens = [0] * n
    for i, s in enumerate(slots):
        lens[s] = rows[i] + cached[i]
    cache, kv = filled(lens, hkv, dh, dt(types[1]), seed, layers=2)
    before = cache.kv.clone()
    cu = [0]
    for r in rows:
        cu.append(cu[-1] + r)
    total = cu[-1] + tail
    g = torch.Generator().manual_seed(seed + 1)
    x = (scale * torch.randn(total, hq + 2 * hkv, dh, generator=g)).to(dt(types[0])).cuda()
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    host = [t.clone().cpu() for t in (q, k, v)]
    gain = [(1 + 0.2 * torch.randn(dh, generator=g)).cuda() if c in gains else None for c in "qk"]
    rope = None
    if rot:
        rope = tuple(torch.randn(PAGE * cache.max_pages, rot // 2, generator=g).cuda() for _ in range(2))
    rule = HeadRule(q_gain=gain[0] if with_q else None, k_gain=gain[1], eps=1e-5, interleaved=interleaved)
    print(f"[heads {types} {heads} rows {rows} rot {rot} {interleaved} {gains}]", flush=True)
    q_out = q if in_place else None
    got = cache.append_heads(1, k, v, i32(slots), i32(cu), rule, q=q if with_q else None, q_out=q_out if with_q else None, rope=rope)
    torch.cuda.synchronize()
    ropeh = None if rope is None else tuple(t.cpu() for t in rope)
    want_kv = before.cpu()
    for i, s in enumerate(slots):
        a, b = cu[i], cu[i + 1]
        pos = torch.arange(cached[i], cached[i] + rows[i])
        if with_q:
            w, m = turned(host[0][a:b], pos, gain[0].cpu() if gain[0] is not None else None, 1e-5, ropeh, interleaved)
            within(got[a:b], w, m, types[0], ("q", i))
        w, m = turned(host[1][a:b], pos, gain[1].cpu() if gain[1] is not None else None, 1e-5, ropeh, interleaved)
        page = cache.page_table[s].cpu().long()[pos // PAGE]
        now = cache.kv.cpu()
        within(now[1, page, 0, :, pos % PAGE], w, m, types[1], ("k", i))
        assert torch.equal(now[1, page, 1, :, pos % PAGE], host[2][a:b].to(dt(types[1]))), ("v", i)
        want_kv[1, page, :, :, pos % PAGE] = now[1, page, :, :, pos % PAGE]
    assert torch.equal(torch.nan_to_num(cache.kv.cpu(), nan=9.0), torch.nan_to_num(want_kv, nan=9.0))  # nothing else
    if with_q and in_place and tail:
        assert torch.equal(got[cu[-1]:].cpu(), host[0][cu[-1]:])


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,rot", [((8, 2, 128), 128), ((5, 1, 128), 48), ((6, 2, 64), 64), ((4, 4, 64), 16), ((3, 1, 64), 0)], ids=str)
def test_layouts(types, interleaved, heads, rot):
    case([1, 17, 0, 33], [0, 15, 4, 100], heads, types, rot, interleaved, "qk", seed=rot)


@pytest.mark.parametrize("gains", ["", "q", "k", "qk"])
@pytest.mark.parametrize("rot", [0, 32, 128])
def test_gains(gains, rot):
    case([2, 40], [9, 0], (8, 4, 128), ("bf16", "bf16"), rot, False, gains)


def test_in_place_and_rows_behind_the_last():
    case([5, 30], [1, 0], (8, 2, 128), ("bf16", "bf16"), 64, True, "qk", tail=3, in_place=True)
    case([5, 30], [1, 0], (8, 2, 64), ("f32", "f32"), 64, False, "qk", tail=3, in_place=True, packed=False)


def test_keys_and_values_alone():
    case([5, 30], [1, 0], (8, 2, 128), ("f32", "bf16"), 96, False, "k", with_q=False)


@pytest.mark.parametrize("scale", [1e-12, 1e-3, 1e18, 1e25])
def test_sizes_of_values(scale):
    """Squares that vanish beside eps, and squares past fp32's range."""
    case([3, 20], [0, 5], (4, 2, 128), ("f32", "f32"), 0, False, "qk", scale=scale)
    case([3, 20], [0, 5], (4, 2, 128), ("bf16", "bf16"), 0, False, "qk", scale=scale)


def test_as_append_without_norms():
    """Half of the dims' layout over the whole head and no gains: the same bits as append."""
    from paper_2605_30852_amd.cache import HeadRule
    from tests.seqcache import PAGE, filled, i32
    for types in TYPES:
        a, _ = filled([30, 7], 2, 128, dt(types[1]), 3)
        b, _ = filled([30, 7], 2, 128, dt(types[1]), 3)
        g = torch.Generator().manual_seed(1)
        x = torch.randn(12, 10, 128, generator=g).to(dt(types[0])).cuda()
        rope = tuple(torch.randn(PAGE * a.max_pages, 64, generator=g).cuda() for _ in range(2))
        args = (0, x[:, 6:8], x[:, 8:], i32([1, 0]), i32([0, 7, 12]))
        qa = a.append(*args, q=x[:, :6], rope=rope)
        qb = b.append_heads(*args, HeadRule(), q=x[:, :6], rope=rope)
        assert torch.equal(qa, qb) and torch.equal(torch.nan_to_num(a.kv, nan=9.0), torch.nan_to_num(b.kv, nan=9.0))


def test_pages_that_are_none_and_sequences_that_are_none():
    """A row whose page the table lacks, a sequence out of range, rows before the first key: nothing is written for them."""
    from paper_2605_30852_amd.cache import HeadRule
    from tests.seqcache import filled, i32
    cache, _ = filled([20, 3, 9, 1], 2, 64, torch.float32, 5)
    cache.page_table[0, 1] = -1
    before = cache.kv.clone()
    x = torch.randn(30, 8, 64, device="cuda")
    gain = torch.ones(64, device="cuda")
    q = cache.append_heads(0, x[:, 4:6], x[:, 6:], i32([0, 7, 1, -1]), i32([0, 6, 10, 20, 30]), HeadRule(q_gain=gain, k_gain=gain), q=x[:, :4],
                           q_out=torch.full((30, 4, 64), 7.0, device="cuda"))
    torch.cuda.synchronize()
    assert (q[6:10] == 7.0).all() and (q[20:] == 7.0).all() and (q[10:17] == 7.0).all() and (q[17:20] != 7.0).any()
    changed = (torch.nan_to_num(cache.kv, nan=9.0) != torch.nan_to_num(before, nan=9.0)).flatten(1).any(0).sum()
    assert changed > 0
    pages = (torch.nan_to_num(cache.kv, nan=9.0) != torch.nan_to_num(before, nan=9.0)).flatten(2).any(-1)[0]
    assert set(pages.nonzero().flatten().tolist()) <= {int(cache.page_table[0, 0]), int(cache.page_table[1, 0])}


def test_in_a_graph():
    """A captured call follows the lengths and the rows on replay, with eager calls in between."""
    from paper_2605_30852_amd.cache import HeadRule
    from tests.seqcache import PAGE, filled, i32
    cache, _ = filled([100, 60], 2, 64, torch.bfloat16, 21)
    other, _ = filled([100, 60], 2, 64, torch.bfloat16, 21)
    g = torch.Generator().manual_seed(2)
    x = torch.randn(5, 8, 64, generator=g).bfloat16().cuda()
    rope = tuple(torch.randn(PAGE * cache.max_pages, 16, generator=g).cuda() for _ in range(2))
    rule = HeadRule(q_gain=torch.rand(64, generator=g).cuda(), k_gain=torch.rand(64, generator=g).cuda())
    seqs, cu = i32([1, 0]), i32([0, 2, 5])

    def call(c):
        return c.append_heads(0, x[:, 4:6], x[:, 6:], seqs, cu, rule, q=x[:, :4], rope=rope)

    call(cache), call(other)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(cache)
    for k in range(4):
        x.copy_(torch.randn(5, 8, 64, generator=g))
        for c in (cache, other):
            c.lens.copy_(i32([100 - 9 * k, 60 - 7 * k]))
        graph.replay()
        want = call(other)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert torch.equal(torch.nan_to_num(cache.kv, nan=9.0), torch.nan_to_num(other.kv, nan=9.0)), k
