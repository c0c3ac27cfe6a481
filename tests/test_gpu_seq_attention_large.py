"""Values near the end of fp32's range whose weighted mean is finite: no sum on the way may be infinite. The scores rise by seven
powers of two behind the first 128 keys, less than what renews a running maximum, and sums of as many values overflow also where no
weight is above one."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]


def large(lens, heads, types, seed, size):
    """A cache of such sequences, with values of `size` to twice that, their keys and values [KV heads][len][dh], and rows of queries."""
    from tests.seqcache import filled
    hq, hkv, dh = heads
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}
    c, kv = filled(lens, hkv, dh, dt[types[1]], seed)
    g = torch.Generator().manual_seed(seed)
    out = []
    for s, n in enumerate(lens):
        k = torch.zeros(n, hkv, dh)
        k[128:, :, 0] = 7.0
        v = size * (1.0 + torch.rand(n, hkv, dh, generator=g))
        v[:, :, 1::3] *= torch.where(torch.rand(n, hkv, (dh + 1) // 3, generator=g) < 0.5, -1.0, 1.0)
        v[:, :, 2::3] /= size
        j = torch.arange(n, device="cuda")
        page = c.page_table[s, j // 16].long()
        for i, x in enumerate((k, v)):
            x = x.to(dt[types[1]])
            c.kv[0][page, i, :, j % 16] = x.cuda()
            out.append(x.transpose(0, 1))
    q = torch.zeros(sum(lens), hq, dh)
    q[:, :, 0] = 0.6931 * dh ** 0.5  # 2^7 of a key's weight between the two kinds
    q[:, :, 1:] = torch.randn(sum(lens), hq, dh - 1, generator=g)
    return c, list(zip(out[::2], out[1::2])), q.to(dt[types[0]])


@pytest.mark.parametrize("size", [1e37, 1.6e38])
@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("heads", [(8, 2, 128), (6, 2, 64), (16, 1, 64)], ids=str)
@pytest.mark.parametrize("max_len", [0, 500])
def test_rows_of_prompts(heads, types, max_len, size):
    """Wide pieces, of two sets of queries and of one, cut and not; the same without a plan."""
    from tests.seqcache import attend, check, i32
    G = heads[0] // heads[1]
    lens, rows = [300, 460, 210, 5000], [100, 32 // G, 3, 2]
    if max_len:
        lens, rows = lens[1:3], [2, 3]
    c, kv, q = large(lens, heads, types, 1, size)
    cu = [0]
    for r in rows:
        cu.append(cu[-1] + r)
    print(f"[large prompt {types} {heads} {max_len} {size}]", flush=True)
    out = c.prompt_attention(0, q[:cu[-1]].cuda(), i32(list(range(len(lens)))), i32(cu), max_len=max_len)
    torch.cuda.synchronize()
    for i, n in enumerate(lens):
        pick = sorted({0, rows[i] // 2, rows[i] - 1})
        want, mag = attend(q[cu[i]:cu[i + 1]][pick], *kv[i], [n - rows[i] + r + 1 for r in pick])
        check(out[cu[i]:cu[i + 1]][pick], want, mag, (types[0], i))


@pytest.mark.parametrize("size", [1e37, 1.6e38])
@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)], ids=str)
def test_rows_behind_a_prefix(heads, types, size):
    """Pieces whose sums a merge joins."""
    from tests.seqcache import agree, attend, check, i32
    n, prefix = 40, 3000
    lens = [prefix + 5 * i for i in range(n)]
    c, kv, q = large(lens, heads, types, 2, size)
    for i in range(1, n):
        agree(c, 0, i, prefix)
    print(f"[large prefix {types} {heads} {size}]", flush=True)
    out = c.prefix_attention(0, q[:n].cuda(), i32(list(range(n))), i32([0, n]), i32([prefix]))
    torch.cuda.synchronize()
    for i in (0, 1, 17, n - 1):
        x = [torch.cat((a[:, :prefix], b[:, prefix:]), 1) for a, b in zip(kv[0], kv[i])]
        want, mag = attend(q[i:i + 1], *x, [lens[i]])
        check(out[i:i + 1], want, mag, (types[0], i))
