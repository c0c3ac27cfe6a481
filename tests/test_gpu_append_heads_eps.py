"""Norms of heads whose squares, or whose eps, lie at the ends of fp32's range, against 64 bits."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("f32", "f32")], ids="-".join)
@pytest.mark.parametrize("scale,eps", [(1e20, 1e38), (1e20, 1e-6), (3e19, 3e38), (1e18, 3.3e38), (1e-3, 3.3e38), (1e-22, 1e-43),
                                       (1e-24, 1e-45), (1e-30, 1e-40), (1e-18, 1e-38), (0.0, 1e-45)])
def test_norms(types, scale, eps):
    """Within 17 roundings of 2^-24 (16 squares of a lane and their joins, half of them in the root, and four more) and the result's own
    half step, 2^-8 or 2^-24."""
    from paper_2605_30852_amd.cache import HeadRule
    from tests.ruled import turned
    from tests.seqcache import PAGE, filled, i32
    for hq, hkv, dh in ((4, 2, 128), (3, 1, 64)):
        cache, _ = filled([20], hkv, dh, dt(types[1]), 51)
        g = torch.Generator().manual_seed(9)
        x = (scale * torch.randn(20, hq + 2 * hkv, dh, generator=g)).to(dt(types[0])).cuda()
        gain = (1 + 0.2 * torch.randn(dh, generator=g)).cuda()
        print(f"[norms {types} {scale} {eps} {dh}]", flush=True)
        q = cache.append_heads(0, x[:, hq:hq + hkv], x[:, hq + hkv:], i32([0]), i32([0, 20]), HeadRule(q_gain=gain, k_gain=gain, eps=eps),
                               q=x[:, :hq])
        pos = torch.arange(20)
        held = torch.tensor(eps, dtype=torch.float32).double().item()
        page = cache.page_table[0].cpu().long()[pos // PAGE]
        for got, y in ((q, x[:, :hq]), (cache.kv.cpu()[0, page, 0, :, pos % PAGE], x[:, hq:hq + hkv])):
            want, mag = turned(y.cpu(), pos, gain.cpu(), held, None, False)
            bound = 17 * 2 ** -24 * mag + (2 ** -8 if got.dtype is torch.bfloat16 else 2 ** -24) * want.abs() + 2.0 ** -133
            assert ((got.double().cpu() - want).abs() <= bound).all(), (types, scale, eps, dh)
