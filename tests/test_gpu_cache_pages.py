"""The pages of a cache of several sequences: growing, forking, truncating and compacting them against lists on the
host, word for word, with the contents that the copies have to carry."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def make(num_pages, max_seqs, max_pages, layers=2, hkv=2, dh=64, dtype="bf16"):
    from paper_2605_30852_amd.cache import PagedCache

    from tests.seqcache import Model
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    c = PagedCache.empty(layers, num_pages, hkv, dh, max_seqs, max_pages, dt)
    g = torch.Generator(device="cuda").manual_seed(num_pages)
    c.kv.normal_(generator=g)
    return c, Model(num_pages, max_seqs, max_pages), c.kv.clone()


def same(c, m, kv0, status, want, what):
    torch.cuda.synchronize()
    assert status.item() == want, (what, status.item(), want)
    assert c.lens.tolist() == m.lens, what
    assert c.refs.tolist() == m.refs, what
    assert c.page_table.tolist() == m.table, what
    assert torch.equal(c.kv, kv0[:, torch.tensor(m.data, device="cuda")]), what


def drive(c, m, kv0, rng, steps):
    from tests.seqcache import i32
    n = len(m.lens)
    for step in range(steps):
        op = rng.choice(["reserve", "reserve", "fork", "truncate", "compact"])
        if op == "compact":
            want = m.compact()
            got = c.compact()
        elif op == "fork":
            empty = [s for s in range(n) if m.lens[s] == 0]
            k = rng.randint(1, max(1, min(4, len(empty))))
            dst = rng.sample(empty, min(k, len(empty))) or [0]
            src = [rng.randrange(n) for _ in dst]
            keep = [rng.randint(0, m.lens[s]) for s in src]
            if rng.random() < 0.1:
                keep[0] = m.lens[src[0]] + 1
            want, got = m.fork(src, dst, keep), c.fork(i32(src), i32(dst), i32(keep))
        else:
            seqs = rng.sample(range(n), rng.randint(1, n))
            if rng.random() < 0.1:
                seqs.append(rng.choice([seqs[0], -1, n]))
                seqs = seqs[-n:]
            if op == "reserve":
                add = [rng.choice([0, 1, 1, 15, 16, 17, rng.randint(0, 60)]) for _ in seqs]
                want, got = m.reserve(seqs, add), c.reserve(i32(seqs), i32(add))
            else:
                keep = [rng.choice([0, 1, 16, rng.randint(0, 100)]) for _ in seqs]
                if rng.random() < 0.1:
                    keep[-1] = -1
                want, got = m.truncate(seqs, keep), c.truncate(i32(seqs), i32(keep))
        same(c, m, kv0, got, want, (step, op))


@pytest.mark.parametrize("pages,seqs,most,dtype,dh", [(40, 6, 8, "bf16", 64), (37, 9, 7, "f32", 128), (700, 40, 33, "bf16", 128), (1, 1, 1, "bf16", 64)])
def test_any_order_of_calls(pages, seqs, most, dtype, dh):
    for seed in range(3):
        c, m, kv0 = make(pages, seqs, most, dtype=dtype, dh=dh)
        drive(c, m, kv0, random.Random(seed), 40)


def test_large_pools_and_batches():
    """More pages than a tile of the plan (16384) and more sequences than its threads (1024)."""
    from tests.seqcache import i32
    c, m, kv0 = make(40000, 1500, 30, layers=1, hkv=1)
    rng = random.Random(5)
    seqs = rng.sample(range(1500), 1500)
    add = [rng.randint(0, 16 * 26) for _ in seqs]
    same(c, m, kv0, c.reserve(i32(seqs), i32(add)), m.reserve(seqs, add), "grow")
    gone = seqs[::3]
    same(c, m, kv0, c.truncate(i32(gone), i32([0] * len(gone))), m.truncate(gone, [0] * len(gone)), "end")
    src = [rng.choice(seqs[1::3]) for _ in gone]
    keep = [m.lens[s] for s in src]
    same(c, m, kv0, c.fork(i32(src), i32(gone), i32(keep)), m.fork(src, gone, keep), "fork")
    one = [1] * len(gone)
    same(c, m, kv0, c.reserve(i32(gone), i32(one)), m.reserve(gone, one), "first tokens")
    same(c, m, kv0, c.compact(), m.compact(), "compact")
    same(c, m, kv0, c.compact(), m.compact(), "compact again")
    too_many = [16 * 30 - n for n in m.lens]
    free = sum(r == 0 for r in m.refs)
    want = m.reserve(list(range(1500)), too_many)
    same(c, m, kv0, c.reserve(i32(list(range(1500))), i32(too_many)), want, ("to the end", free))


def test_a_captured_step_follows_the_state():
    """Reserve and truncate in a graph: each replay acts on the state that the last one left."""
    from tests.seqcache import i32
    c, m, kv0 = make(60, 5, 12)
    seqs, add, two, keep = [3, 0, 4], [7, 1, 20], [1, 2], [5, 0]
    a, b, d, e = i32(seqs), i32(add), i32(two), i32(keep)
    c.reserve(a, b), c.truncate(d, e), c.compact()
    m.reserve(seqs, add), m.truncate(two, keep), m.compact()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s1, s2, s3 = c.reserve(a, b), c.truncate(d, e), c.compact()
    for i in range(8):
        g.replay()
        want = m.reserve(seqs, add), m.truncate(two, keep), m.compact()
        same(c, m, kv0, s3, want[2], i)
        assert (s1.item(), s2.item()) == want[:2]
        more = c.reserve(d, i32([3, 3]))  # eager work between the replays
        same(c, m, kv0, more, m.reserve(two, [3, 3]), ("eager", i))
