"""Equal scores under a cap in neighbouring tiles, one of which holds a score of another range and so takes another formula."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]


def dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


@pytest.mark.parametrize("swap", [False, True])
@pytest.mark.parametrize("cap", [60.0, 100.0, 200.0, 500.0])
@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_equal_scores(types, cap, swap):
    """Two tiles of 64 keys of one score, values of 1 and -1 whose mean is 0; the first key of each has a far lower score, in one of them
    past what the others' formula takes. The same formula, or others that differ by less than 1e-3 in a score, give probabilities that
    round to the same bf16 numbers, 1 (fp32 ones differ by 1e-3 of themselves): outputs within half of 1e-3, and 2^-10 holds that
    with what the low scores weigh, e^-36."""
    from tests.seqcache import filled, i32
    from paper_2605_30852_amd.cache import AttentionRule
    hq, hkv, dh, new = 4, 1, 64, 64
    for x in (0.1, 0.25, 0.4, 0.5, 0.6, 0.75, 0.85):
        cache, _ = filled([128 + new], hkv, dh, dt(types[1]), 41)
        far, near = (-0.7, -0.4) if x <= 0.5 else (-0.97, -0.5)
        k = torch.zeros(128 + new, dh)
        v = torch.zeros(128 + new, dh)
        a, b = (64, 0) if swap else (0, 64)
        k[:128, 0], k[a, 0], k[b, 0], k[128:, 0] = x, far, near, -0.4
        v[a + 1:a + 64], v[b + 1:b + 64] = 1.0, -1.0
        k[:, 0] *= cap / 2  # a score is 2 of it
        j = torch.arange(128 + new, device="cuda")
        page = cache.page_table[0].long()[j // 16]
        cache.kv[0, page, 0, 0, j % 16] = k.to(dt(types[1])).cuda()
        cache.kv[0, page, 1, 0, j % 16] = v.to(dt(types[1])).cuda()
        q = torch.zeros(new, hq, dh, dtype=dt(types[0]), device="cuda")
        q[..., 0] = 16.0
        for slopes in (None, [0.0] * hq):
            out = cache.prompt_attention(0, q, i32([0]), i32([0, new]), rule=AttentionRule(
                cap=cap, slopes=torch.tensor(slopes, device="cuda") if slopes else None))
            worst = out.double().abs().max().item()
            print(f"[{types} cap {cap} x {x} {worst:.2e}]", flush=True)
            assert worst <= 2 ** -10, (types, cap, x, worst)
