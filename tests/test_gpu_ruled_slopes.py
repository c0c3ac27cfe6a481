"""The steepest slopes that fp32 holds: a row's nearest key counts alone."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]


def dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


@pytest.mark.parametrize("cap", [0.0, 7.0, 100.0])
@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_steepest(types, cap):
    """Whole and split pieces, one launch of few queries, decode rows with and without a shared prefix."""
    from paper_2605_30852_amd.cache import AttentionRule
    from tests.ruled import attend, check
    from tests.seqcache import agree, filled, i32
    hq, hkv, dh = 4, 2, 64
    top = torch.finfo(torch.float32).max
    slopes = [top, 2.4e38, 1e38, 1e30]
    g = torch.Generator().manual_seed(3)
    rule = AttentionRule(cap=cap, slopes=torch.tensor(slopes, device="cuda"))
    for n, new, max_len in ((70, 70, 0), (70, 5, 70), (1500, 40, 0)):
        cache, kv = filled([n], hkv, dh, dt(types[1]), 61)
        q = (1.5 * torch.randn(new, hq, dh, generator=g)).to(dt(types[0])).cuda()
        print(f"[steepest {types} {cap} {n} {new}]", flush=True)
        out = cache.prompt_attention(0, q, i32([0]), i32([0, new]), max_len=max_len, rule=rule)
        want, mag = attend(q, kv[0][0, 0], kv[0][0, 1], [(n - new + r, 0, 0) for r in range(new)], cap, slopes)
        check(out, want, mag, (types[0], n, new))
    lens = [600 + i for i in range(20)]
    cache, kv = filled(lens, hkv, dh, dt(types[1]), 62)
    for i in range(1, 20):
        agree(cache, 0, i, 600)
    q = (1.5 * torch.randn(20, hq, dh, generator=g)).to(dt(types[0])).cuda()
    for groups in ((), (i32([0, 20]), i32([600]))):
        out = cache.prefix_attention(0, q, i32(list(range(20))), *groups, rule=rule)
        for i in range(20):
            x = torch.cat([kv[0][0, :, :, :600], kv[i][0, :, :, 600:]], 2)
            want, mag = attend(q[i:i + 1], x[0], x[1], [(lens[i] - 1, 0, 0)], cap, slopes)
            check(out[i:i + 1], want, mag, (types[0], "row", i, len(groups)))
