"""Rotary tables against exact angles: every scaling, odd sizes, positions far from 0, streams, graphs."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SCALINGS = [("", 1.0, 0), ("linear", 4.0, 0), ("linear", 0.5, 0), ("ntk", 8.0, 0), ("parts", 8.0, 4096)]


def compare(freq, cos, sin, first, amplitude, positions):
    """Each value is rounded once, 2^-24 of it, from 64 bits whose angle is off by some 2^-54 of a turn, 2^-51."""
    from tests.ruled import cos_sin
    for r in positions:
        for i in range(len(freq)):
            want = cos_sin(first + r, float(freq[i]), amplitude)
            for got, w in zip((cos[r, i].item(), sin[r, i].item()), want):
                assert abs(got - w) <= 2 ** -24 * abs(w) * 1.0001 + 2 ** -51 * abs(amplitude), (first + r, i, got, w)


@pytest.mark.parametrize("scaling", SCALINGS, ids=str)
@pytest.mark.parametrize("dims", [4, 6, 16, 64, 112, 128, 256])
def test_tables(dims, scaling):
    from paper_2605_30852_amd.rope import RopeScaling, rope_frequencies, rope_table
    kind, factor, original = scaling
    f = rope_frequencies(dims, 500000.0, RopeScaling(kind, factor, original, 1.0, 4.0) if kind else None)
    rng = random.Random(dims)
    for n, first, amplitude in ((1, 0, 1.0), (7, 3, 1.3), (300, 131000, 0.9)):
        cos, sin = rope_table(f, n, first=first, amplitude=amplitude)
        assert cos.shape == sin.shape == (n, dims // 2) and cos.dtype == torch.float32
        compare(f, cos.cpu(), sin.cpu(), first, amplitude, {0, n - 1, rng.randrange(n), rng.randrange(n)})


@pytest.mark.parametrize("first", [-5, 1 << 24, (1 << 30) - 9, 1 << 30, -(1 << 30)])
def test_far_positions(first):
    from paper_2605_30852_amd.rope import rope_frequencies, rope_table
    f = rope_frequencies(64, 10000.0)
    cos, sin = rope_table(f, 9, first=first)
    compare(f, cos.cpu(), sin.cpu(), first, 1.0, range(9))


def test_frequencies_of_the_callers_own():
    from paper_2605_30852_amd.rope import rope_table
    f = torch.tensor([0.0, -0.3, 1e3, 1e-12, 3.0], dtype=torch.float64)
    cos, sin = rope_table(f, 40, first=100000)
    compare(f, cos.cpu(), sin.cpu(), 100000, 1.0, range(40))


def test_every_row_of_a_large_table_and_into_out():
    """Against double precision on the device, whose angles are off by 2^-53 of themselves: 200000 radians by 2.3e-11."""
    from paper_2605_30852_amd.rope import rope_frequencies, rope_table
    for dims in (128, 80, 6):
        f = rope_frequencies(dims, 10000.0)
        n = 200003
        out = (torch.full((n, dims // 2), 7.0, device="cuda"), torch.full((n, dims // 2), 7.0, device="cuda"))
        got = rope_table(f, n, out=out)
        assert got[0] is out[0] and got[1] is out[1]
        ang = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * f.cuda()
        for x, w in zip(out, (ang.cos(), ang.sin())):
            assert ((x.double() - w).abs() <= 2 ** -24 * w.abs() + 1e-10).all()


def test_no_positions_and_other_streams():
    from paper_2605_30852_amd.rope import rope_frequencies, rope_table
    f = rope_frequencies(32, 10000.0)
    assert rope_table(f, 0)[0].shape == (0, 16)
    want = rope_table(f, 500)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = rope_table(f, 500)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_in_a_graph():
    """The frequencies travel with the launch: what the host does with them afterwards does not matter."""
    from paper_2605_30852_amd.rope import rope_frequencies, rope_table
    f = rope_frequencies(64, 10000.0)
    want = [x.clone() for x in rope_table(f, 77, first=5)]
    out = (torch.empty(77, 32, device="cuda"), torch.empty(77, 32, device="cuda"))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rope_table(f, 77, first=5, out=out)
    f.zero_()
    for _ in range(3):
        out[0].zero_(), out[1].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
