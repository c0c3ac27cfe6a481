"""Which keys a row attends, counted: queries of zeros weigh all keys alike, and key j's value is one at place j % head_dim and zero
elsewhere, so an output times the number of keys is how many of them have its place. Weights and sums are whole numbers, which bf16 and
fp32 hold; what rounds is the output, by half a step of its type. A place has at most 100 keys, of which bf16's half step is 0.4: a
key left out or taken twice, one more or less, is always seen."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def counting(lens, hkv, dh, dtype, seed):
    """Keys of noise with such values."""
    from tests.seqcache import filled
    c, _ = filled(lens, hkv, dh, DT[dtype], seed)
    for s, n in enumerate(lens):
        j = torch.arange(n, device="cuda")
        v = torch.nn.functional.one_hot(j % dh, dh).to(DT[dtype])
        c.kv[0][c.page_table[s, j // 16].long(), 1, :, j % 16] = v[:, None].expand(n, hkv, dh)
    return c


def expect(out, limits, what):
    """out [rows][heads][dh], row i over its first limits[i] keys."""
    dh, most = out.shape[-1], max(max(limits), 1)
    j = torch.arange(most, device="cuda")
    counts = torch.cat((torch.zeros(1, dh, device="cuda"), torch.nn.functional.one_hot(j % dh, dh).cumsum(0))).double()
    assert counts.max() <= 100
    n = torch.tensor(limits, device="cuda").clamp(min=0)
    want = counts[n][:, None]
    got = out.double() * n.clamp(min=1)[:, None, None]
    # the output's half step, and fp32's for the reciprocal and the product
    bound = want * (torch.finfo(out.dtype).eps / 2 + 2 * 2 ** -24)
    worst = ((got - want).abs() - bound).max().item()
    assert worst <= 0.0, (what, worst)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("heads", [(8, 2, 128), (32, 8, 128), (6, 2, 64), (4, 4, 64), (16, 1, 128)], ids=str)
def test_prompts(heads, types):
    """Every row of prompts whose tiles, steps and pages end at odd places, behind no keys and behind some."""
    from tests.seqcache import i32
    hq, hkv, dh = heads
    G = hq // hkv
    rpt = 128 // G
    rows, cached = [3 * rpt + 1, 2 * rpt, 65, 33, 17, 1, 5], [0, 1, 63, 500, 15, 1000, 777]
    lens = [r + c for r, c in zip(rows, cached)]
    c = counting(lens, hkv, dh, types[1], 1)
    cu = [0]
    for r in rows:
        cu.append(cu[-1] + r)
    q = torch.zeros(cu[-1], hq, dh, dtype=DT[types[0]], device="cuda")
    print(f"[keys of prompts {types} {heads}]", flush=True)
    out = c.prompt_attention(0, q, i32(list(range(len(rows)))), i32(cu))
    for i, n in enumerate(rows):
        expect(out[cu[i]:cu[i + 1]], [cached[i] + r + 1 for r in range(n)], (types, "sequence", i))


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("heads", [(8, 2, 128), (6, 2, 64)], ids=str)
@pytest.mark.parametrize("rows,cached", [([40, 3], [5003, 4001]), ([2], [5119]), ([50], [2500]), ([3, 7, 1], [4096, 4100, 4095])], ids=str)
def test_long_caches(heads, types, rows, cached):
    """Pieces of long caches, cut."""
    from tests.seqcache import i32
    hq, hkv, dh = heads
    lens = [r + c for r, c in zip(rows, cached)]
    cu = [0]
    for r in rows:
        cu.append(cu[-1] + r)
    q = torch.zeros(cu[-1], hq, dh, dtype=DT[types[0]], device="cuda")
    print(f"[keys of long caches {types} {heads} {rows} {cached}]", flush=True)
    c = counting(lens, hkv, dh, types[1], 2)
    out = c.prompt_attention(0, q, i32(list(range(len(rows)))), i32(cu))
    for i, n in enumerate(rows):
        expect(out[cu[i]:cu[i + 1]], [cached[i] + r + 1 for r in range(n)], (types, "sequence", i))


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)], ids=str)
@pytest.mark.parametrize("prefix", [1, 15, 16, 17, 250, 257, 1000, 2047])
def test_prefixes(heads, types, prefix):
    """Rows behind a prefix that ends anywhere in a page, rows shorter than it, rows of their own."""
    from tests.seqcache import i32
    hq, hkv, dh = heads
    n = 37
    lens = [prefix + (7 * i) % 40 for i in range(n)] + [prefix // 2, 0, 100, prefix + 300]
    c = counting(lens, hkv, dh, types[1], 3)  # the sequences agree in all keys that they share
    q = torch.zeros(len(lens), hq, dh, dtype=DT[types[0]], device="cuda")
    print(f"[keys of prefixes {types} {heads} {prefix}]", flush=True)
    for cu, plens in (([0, n + 2, n + 4], [prefix, 0]), ([0, 9, n, n + 4], [prefix, prefix, min(prefix, 100)])):
        out = c.prefix_attention(0, q, i32(list(range(len(lens)))), i32(cu), i32(plens))
        expect(out, lens, (types, prefix, cu))


@pytest.mark.parametrize("heads,rows,cached", [((128, 8, 64), [700, 1, 450], [0, 70, 333]), ((64, 8, 128), [1, 2300, 33], [5, 0, 1000]),
                                               ((96, 16, 128), [1500, 15], [7, 0])], ids=str)
def test_rows_at_the_edges_of_tiles(heads, rows, cached):
    """Batches of many rows: those on both sides of every edge of their tiles, odd ones too, against 64 bits."""
    from tests.seqcache import attend, check, filled, i32
    hq, hkv, dh = heads
    lens = [r + c for r, c in zip(rows, cached)]
    cache, kv = filled(lens, hkv, dh, torch.bfloat16, 21)
    cu = [0]
    for r in rows:
        cu.append(cu[-1] + r)
    q = (1.5 * torch.randn(cu[-1], hq, dh, generator=torch.Generator().manual_seed(22))).bfloat16()
    out = cache.prompt_attention(0, q.cuda(), i32(list(range(len(rows)))), i32(cu)).cpu()
    rpt = 128 // (hq // hkv)
    for i, n in enumerate(rows):
        edges = [e for e in range(rpt, n, rpt)]
        edges = edges[:3] + edges[-3:]
        pick = sorted({r for e in edges for r in (e - 1, e)} | {0, n - 1})
        want, mag = attend(q[cu[i]:cu[i + 1]][pick], kv[i][0, 0], kv[i][0, 1], [cached[i] + r + 1 for r in pick])
        check(out[cu[i]:cu[i + 1]][pick], want, mag, ("bf16", i))
