"""Scores under a cap that rise with the distance (slopes below 0), as far as fp32's range and past it, against 64 bits: the sum of a
row's probabilities may leave that range while its outputs, of mixed signs or small values, do not."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]
CAP = 7.0


def dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def rising(heads):
    """A row of key p has exponents up to -slope p log2(e) + 10 beside an offset of -16: they pass 2^128 from some 3550, 1770 and 1140
    keys on, and stay below it at half of the slope."""
    return [(-0.02, -0.04, -0.0625, -0.01)[h % 4] for h in range(heads)]


def check(got, want, mag, what):
    """What a score, in units of its own, may be off by: its 64 products 8e-6; a cap's tanh 2.4e-6 (bf16 rows: four terms, 4e-5 of a score
    of 7, 2.8e-4); the distance times its slope, up to 370 in units of log2, by half a step of [256, 512), 2^-16, in a row that is made
    again, and as much in the change of units, 2.6e-5 (others stay below 128: five roundings of 2^-18, 1.3e-5); the slope, two
    roundings of 2^-24 times the spread of the distances that count, 25, 3e-6. A probability moves by twice the 4e-5: 1e-4 (and 6e-4) of
    sum p |v|. bf16 rows: half a step, 2^-8, of each rounded probability and of the output."""
    got = got.double().cpu()
    assert torch.isfinite(got).all(), what
    bound = 1e-4 * mag + 1e-30
    if what[0] == "bf16":
        bound = bound + 6e-4 * mag + 2 ** -8 * (want.abs() + 1.01 * mag)
    worst = ((got - want).abs() / bound).max().item()
    assert worst <= 1.0, (what, worst)


def scaled(cache, kv, factor):
    """The values of every sequence, times factor (a power of two)."""
    cache.kv[:, :, 1] *= factor
    return [torch.stack([x[0, 0], x[0, 1] * factor]) for x in kv]


def rule_of(slopes, **kw):
    from paper_2605_30852_amd.cache import AttentionRule
    return AttentionRule(cap=CAP, slopes=torch.tensor(slopes, device="cuda"), **kw)


@pytest.mark.parametrize("factor", [1.0, 2.0 ** -6])
@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_whole_pieces(types, factor):
    """A prompt of so many tiles that none is split."""
    from tests.ruled import attend
    from tests.seqcache import filled, i32
    n, hq, hkv, dh = 4000, 32, 8, 64
    cache, kv = filled([n], hkv, dh, dt(types[1]), 31)
    x = scaled(cache, kv, factor)[0]
    q = (1.5 * torch.randn(n, hq, dh, generator=torch.Generator().manual_seed(7))).to(dt(types[0])).cuda()
    slopes = rising(hq)
    print(f"[rising, whole {types} {factor}]", flush=True)
    out = cache.prompt_attention(0, q, i32([0]), i32([0, n]), rule=rule_of(slopes))
    rows = [*range(1120, 1210, 6), *range(1740, 1870, 8), *range(3500, 3760, 16), 3, n - 1]
    want, mag = attend(q[rows], x[0], x[1], [(r, 0, 0) for r in rows], CAP, slopes)
    check(out[rows], want, mag, (types[0], factor))


@pytest.mark.parametrize("factor", [1.0, 2.0 ** -6])
@pytest.mark.parametrize("cached", [1120, 1770, 3560, 3680])
@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_split_pieces(types, cached, factor):
    """Few rows behind a long cache: the far keys, which count, are pieces of their own."""
    from tests.ruled import attend
    from tests.seqcache import filled, i32
    new, hq, hkv, dh = 60, 4, 2, 64
    cache, kv = filled([cached + new], hkv, dh, dt(types[1]), 32)
    x = scaled(cache, kv, factor)[0]
    q = (1.5 * torch.randn(new, hq, dh, generator=torch.Generator().manual_seed(7))).to(dt(types[0])).cuda()
    for slopes in (rising(hq), [-0.02] * hq, [-0.04, -0.0625] * 2):
        print(f"[rising, split {types} {cached} {factor} {slopes}]", flush=True)
        for kw in ({}, dict(open_lens=i32([40]), window=cached - 100)):
            out = cache.prompt_attention(0, q, i32([0]), i32([0, new]), rule=rule_of(slopes, **kw))
            sees = [(cached + r, 0, 40 if kw else 0) for r in range(0, new, 3)]
            want, mag = attend(q[::3], x[0], x[1], sees, CAP, slopes, kw.get("window", 0))
            check(out[::3], want, mag, (types[0], cached, factor, bool(kw)))


@pytest.mark.parametrize("factor", [1.0, 2.0 ** -6])
@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_a_group_that_shares_its_far_keys(types, factor):
    from tests.ruled import attend
    from tests.seqcache import agree, filled, i32
    rows, hq, hkv, dh = 20, 4, 2, 64
    for prefix in (1130, 1790, 3600, 3700):
        lens = [prefix + 7 * i for i in range(rows)]
        cache, kv = filled(lens, hkv, dh, dt(types[1]), 33)
        x = scaled(cache, kv, factor)
        for i in range(1, rows):
            agree(cache, 0, i, prefix)
        q = (1.5 * torch.randn(rows, hq, dh, generator=torch.Generator().manual_seed(8))).to(dt(types[0])).cuda()
        slopes = rising(hq)
        print(f"[rising, group {types} {prefix} {factor}]", flush=True)
        out = cache.prefix_attention(0, q, i32(list(range(rows))), i32([0, rows]), i32([prefix]), rule=rule_of(slopes))
        for i in range(rows):
            y = torch.cat([x[0][:, :, :prefix], x[i][:, :, prefix:]], 2)
            want, mag = attend(q[i:i + 1], y[0], y[1], [(lens[i] - 1, 0, 0)], CAP, slopes)
            check(out[i:i + 1], want, mag, (types[0], prefix, i))
