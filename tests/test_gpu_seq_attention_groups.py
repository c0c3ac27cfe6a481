"""Groups of rows that do not ascend: no row shares anything, every row's own pages are read."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")], ids="-".join)
@pytest.mark.parametrize("heads", [(8, 2, 128), (32, 8, 128), (3, 1, 64)], ids=str)
def test_groups_that_do_not_ascend(heads, types):
    from tests.seqcache import attend, check, filled, i32
    hq, hkv, dh = heads
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}
    rng = random.Random(1)
    n = 40
    lens = [rng.choice([0, 5, 40, 300, 700]) for _ in range(n)]
    cache, kv = filled(lens, hkv, dh, dt[types[1]], 1)
    q = (1.5 * torch.randn(n, hq, dh, generator=torch.Generator().manual_seed(2))).to(dt[types[0]]).cuda()
    want, mag = zip(*(attend(q[i:i + 1], kv[i][0, 0], kv[i][0, 1], [lens[i]]) for i in range(n)))
    for cu in ([n if i % 2 else 0 for i in range(n + 1)], [0 if i % 2 else n for i in range(n + 1)], [rng.randint(0, n) for _ in range(n + 1)],
               [0, n, n - 1, n], list(range(n, -1, -1)), [-9, n + 9, 4, 1 << 30]):
        print(f"[groups {types} {heads} {cu}]", flush=True)
        out = cache.prefix_attention(0, q, i32(list(range(n))), i32(cu), i32([600] * (len(cu) - 1)))
        torch.cuda.synchronize()
        check(out, torch.cat(want), torch.cat(mag), (types[0], cu))
