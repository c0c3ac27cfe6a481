"""Queries rotated in place: the same as into other memory."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_in_place(dtype):
    from paper_2605_30852_amd import binding as B
    from tests.seqcache import filled, i32
    from tests.test_gpu_cache_serving import rope_table
    c, _ = filled([40, 7], 2, 64, torch.bfloat16, 1, stale=0.0)
    rope = tuple(t.cuda() for t in rope_table(16 * c.max_pages, 64))
    x = torch.randn(9, 8, 64, generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    args = (i32([1, 0]), i32([0, 4, 9]))
    y = x.clone()
    want = c.append(0, x[:, 4:6], x[:, 6:], *args, q=x[:, :4], rope=rope)
    kv = c.kv.clone()
    assert torch.equal(x, y)
    got = c.append(0, y[:, 4:6], y[:, 6:], *args, q=y[:, :4], q_out=y[:, :4], rope=rope)
    assert torch.equal(got, want) and torch.equal(y[:, 4:], x[:, 4:]) and torch.equal(c.kv, kv)
    flat = x.view(-1)
    tight = flat[:9 * 4 * 64].view(9, 4, 64)  # from the same address, other strides
    with pytest.raises(B.SPDError, match="the same stride"):
        c.append(0, x[:, 4:6], x[:, 6:], *args, q=x[:, :4], q_out=tight, rope=rope)
    one = x[:1, :4].clone()
    c.append(0, x[:1, 4:6], x[:1, 6:], i32([1]), i32([0, 1]), q=one, q_out=one.as_strided((1, 4, 64), (999, 64, 1)), rope=rope)
    assert torch.equal(one, c.append(0, x[:1, 4:6], x[:1, 6:], i32([1]), i32([0, 1]), q=x[:1, :4], rope=rope))
