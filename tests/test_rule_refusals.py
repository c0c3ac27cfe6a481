"""What the calls under rules refuse, on the host, before anything is launched (the pointers here are never dereferenced), and the
frequencies, which are computed there."""
import ctypes as ct

import pytest

from paper_2605_30852_amd import binding as B
from tests.test_cache_refusals import BAD_CACHES, BIG, cache, refused


def head_rule(**kw):
    d = dict(q_gain=128, k_gain=144, eps=1e-6, rot=128, interleaved=0)
    d.update(kw)
    return B.spd_head_rule(*[d[k] for k, _ in B.spd_head_rule._fields_])


def append_heads(c=None, **kw):
    d = dict(layer=0, k=16, k_stride=256, v=32, v_stride=256, q=48, q_stride=1024, q_out=64, q_out_stride=1024, n_q_heads=8,
             dtype=B.SPD_BF16, rule=head_rule(), rope_cos=80, rope_sin=96, rope_positions=80, seqs=4, cu_rows=8, nseqs=2, rows=3, stream=0)
    d.update(kw)
    B.spd_cache_append_heads(c or cache(), **d)


def rule(**kw):
    d = dict(cap=30.0, window=5, slopes=16, first=20, open_lens=24)
    d.update(kw)
    return B.spd_attention_rule(*[d[k] for k, _ in B.spd_attention_rule._fields_])


def prompt(c=None, **kw):
    d = dict(layer=0, q=16, q_stride=1024, out=32, out_stride=1024, n_q_heads=8, dtype=B.SPD_BF16, seqs=4, cu_rows=8, nseqs=2,
             rows=3, max_len=0, rule=rule(), workspace=256, ws_bytes=BIG, stream=0)
    d.update(kw)
    B.spd_prompt_attention_ruled(c or cache(), **d)


def prefix(c=None, **kw):
    d = dict(layer=0, q=16, q_stride=1024, out=32, out_stride=1024, n_q_heads=8, dtype=B.SPD_BF16, seqs=4, nseqs=2, cu_groups=8,
             prefix_lens=12, ngroups=1, max_len=0, rule=rule(), workspace=256, ws_bytes=BIG, stream=0)
    d.update(kw)
    B.spd_prefix_attention_ruled(c or cache(), **d)


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_a_bad_cache(bad):
    if bad != dict(refs=0):
        refused(append_heads, cache(**bad))
        refused(prompt, cache(**bad))
        refused(prefix, cache(**bad))


@pytest.mark.parametrize("bad", [dict(layer=2), dict(layer=-1), dict(k=0), dict(v=36), dict(k_stride=250), dict(q=0), dict(q_out=0),
                                 dict(n_q_heads=0), dict(dtype=3), dict(rope_cos=0), dict(rope_sin=100), dict(rope_positions=79),
                                 dict(seqs=0), dict(cu_rows=2), dict(nseqs=0), dict(nseqs=5), dict(rows=-1), dict(rows=1 << 24),
                                 dict(q=64, q_out=64, q_out_stride=1032)], ids=str)
def test_append_heads(bad):
    refused(append_heads, **bad)


@pytest.mark.parametrize("bad", [dict(q_gain=132), dict(k_gain=8), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("inf")),
                                 dict(eps=float("nan")), dict(rot=8), dict(rot=24), dict(rot=144), dict(rot=-16), dict(rot=0),
                                 dict(interleaved=2), dict(interleaved=-1)], ids=str)
def test_head_rules(bad):
    refused(append_heads, rule=head_rule(**bad))


def test_head_rules_that_need_something():
    refused(append_heads, q=0, q_out=0, n_q_heads=0)  # a gain of queries that are not there
    refused(append_heads, rope_cos=0, rope_sin=0, rope_positions=0)  # dims to turn, and no table
    with pytest.raises(B.SPDError):
        B._check("", B.lib().spd_cache_append_heads(ct.byref(cache()), 0, 16, 256, 32, 256, 48, 1024, 64, 1024, 8, B.SPD_BF16, None, 80, 96,
                                                    80, 4, 8, 2, 3, 0))
    append_heads(rows=0)  # nothing


@pytest.mark.parametrize("bad", [dict(layer=2), dict(q=0), dict(q=24), dict(out=16), dict(out_stride=1020), dict(n_q_heads=3),
                                 dict(n_q_heads=34), dict(dtype=2), dict(seqs=0), dict(seqs=6), dict(nseqs=0), dict(max_len=-1),
                                 dict(workspace=0), dict(workspace=128)], ids=str)
def test_attention(bad):
    refused(prompt, **bad)
    refused(prefix, **bad)


@pytest.mark.parametrize("bad", [dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=1e-7), dict(cap=2e6),
                                 dict(window=-1), dict(slopes=2), dict(first=5), dict(open_lens=6)], ids=str)
def test_attention_rules(bad):
    refused(prompt, rule=rule(**bad))
    refused(prefix, rule=rule(**bad))


def test_attention_of_one_kind():
    refused(prompt, cu_rows=0)
    refused(prompt, rows=-1)
    refused(prefix, nseqs=4097)
    refused(prefix, cu_groups=0)
    refused(prefix, prefix_lens=0)
    refused(prefix, ngroups=3)
    refused(prompt, ws_bytes=0, code=B.SPD_E_CAPACITY)
    refused(prefix, ws_bytes=0, code=B.SPD_E_CAPACITY)
    for f, a in ((B.lib().spd_prompt_attention_ruled, (0, 16, 1024, 32, 1024, 8, 1, 4, 8, 2, 3, 0, None, 256, BIG, 0)),
                 (B.lib().spd_prefix_attention_ruled, (0, 16, 1024, 32, 1024, 8, 1, 4, 2, 8, 12, 1, 0, None, 256, BIG, 0))):
        assert f(ct.byref(cache()), *a) == B.SPD_E_INVAL  # no rule
    prompt(rows=0)  # nothing


def test_rope():
    from tests.ruled import frequencies
    S = B.spd_rope_scaling
    for dims, base in ((128, 10000.0), (2, 500000.0), (256, 1.5)):
        for s, ref in ((None, ()), (S(B.SPD_ROPE_LINEAR, 0, 4.0, 0, 0), ("linear", 4.0)), (S(B.SPD_ROPE_BASE, 0, 4.0, 0, 0), ("ntk", 4.0)),
                       (S(B.SPD_ROPE_PARTS, 4096, 8.0, 1.0, 32.0), ("parts", 8.0, 4096, 1.0, 32.0))):
            if dims == 2 and s is not None and s.kind == B.SPD_ROPE_BASE:
                continue
            for got, want in zip(B.spd_rope_frequencies(dims, base, s), frequencies(dims, base, *ref)):
                assert abs(got - want) <= 1e-13 * want  # two ways to a power, some roundings of 2^-53 times log(base)
    for bad in ((3, 1e4, None), (0, 1e4, None), (258, 1e4, None), (1 << 30, 1e4, None), (-2, 1e4, None), (64, 1.0, None), (64, float("inf"), None), (64, float("nan"), None),
                (64, 1e4, S(4, 0, 2.0, 0, 0)), (64, 1e4, S(-1, 0, 2.0, 0, 0)), (64, 1e4, S(1, 0, 0.0, 0, 0)), (64, 1e4, S(1, 0, float("nan"), 0, 0)),
                (2, 1e4, S(2, 0, 2.0, 0, 0)), (64, 1e4, S(3, 0, 2.0, 1.0, 4.0)), (64, 1e4, S(3, 9, 2.0, 4.0, 4.0)),
                (64, 1e4, S(3, 9, 2.0, 1.0, float("inf")))):
        refused(B.spd_rope_frequencies, *bad)
    f = (ct.c_double * 4)(1.0, 0.5, 0.1, 0.0)

    def table(freq=f, pairs=4, first=0, positions=3, amplitude=1.0, cos=16, sin=32):
        B.spd_rope_table(freq, pairs, first, positions, amplitude, cos, sin, 0)

    for bad in (dict(pairs=0), dict(pairs=129), dict(positions=-1), dict(first=(1 << 30) + 1), dict(first=-(1 << 30) - 1),
                dict(amplitude=float("nan")), dict(cos=0), dict(sin=8), dict(freq=None),
                dict(freq=(ct.c_double * 4)(1.0, float("nan"), 0, 0)), dict(freq=(ct.c_double * 4)(1.0, 0, 0, 1001.0))):
        refused(table, **bad)
    table(positions=0, cos=0, sin=0)  # nothing


def test_rules_of_the_python_classes():
    torch = pytest.importorskip("torch")
    from paper_2605_30852_amd.cache import AttentionRule, HeadRule
    from paper_2605_30852_amd.rope import RopeScaling, rope_frequencies, rope_table
    for bad in (dict(cap=-1.0), dict(cap=float("nan")), dict(window=-1), dict(window=1 << 31), dict(slopes=torch.ones(4)),
                dict(first=torch.ones(4, dtype=torch.int32)), dict(open_lens=torch.ones(4, dtype=torch.int64))):
        with pytest.raises(ValueError):
            AttentionRule(**bad)
    with pytest.raises(ValueError):
        HeadRule(q_gain=torch.ones(64))
    with pytest.raises(ValueError):
        rope_frequencies(64, 1e4, RopeScaling("other", 2.0))
    with pytest.raises(ValueError):
        rope_table(torch.ones(4), 5)
    with pytest.raises(ValueError):
        rope_table(torch.ones(4, dtype=torch.float64), -1)
