"""Children of any number and length, in tables of any width, whichever launches they take."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,most,width", [(1, 130, 130), (1, 5000, 5000), (2, 9000, 13000), (3, 3000, 4096), (3, 3000, 4097), (5, 2000, 2400),
                                          (7, 1500, 1700), (15, 700, 800), (16, 40, 768), (17, 700, 722), (17, 700, 723), (64, 60, 192),
                                          (64, 190, 193), (65, 60, 180), (130, 20, 94), (300, 3, 40)], ids=str)
def test_children(n, most, width):
    from tests.seqcache import i32
    from tests.test_gpu_cache_pages import make, same
    rng = random.Random(n)
    parents = min(n, 3)
    c, m, kv0 = make(parents * most + 9, n + parents, width, layers=1, hkv=1)
    who = list(range(parents))
    add = [16 * most - rng.randint(0, 15)] + [rng.randint(0, 16 * most) for _ in who[1:]]
    same(c, m, kv0, c.reserve(i32(who), i32(add)), m.reserve(who, add), "parents")
    src = [rng.choice(who) for _ in range(n)]
    src[0] = 0
    dst = rng.sample(range(parents, parents + n), n)
    keep = [rng.choice([m.lens[s], rng.randint(0, m.lens[s])]) for s in src]
    keep[0] = m.lens[0]
    print(f"[fork {n} children of up to {most} pages, {width} wide]", flush=True)
    for bad in ([m.lens[src[-1]] + 1], [-1]):
        same(c, m, kv0, c.fork(i32(src), i32(dst), i32(keep[:-1] + bad)), m.fork(src, dst, keep[:-1] + bad), "a length")
    same(c, m, kv0, c.fork(i32(src), i32(dst), i32(keep)), m.fork(src, dst, keep), "fork")
    same(c, m, kv0, c.fork(i32(src), i32(dst), i32([0] * n)), m.fork(src, dst, [0] * n), "children that are there")
    cut = [rng.randint(0, k) for k in keep]
    same(c, m, kv0, c.truncate(i32(dst), i32(cut)), m.truncate(dst, cut), "cut")
