"""What the calls on a cache of several sequences refuse, on the host, before anything is launched (the pointers here
are never dereferenced)."""
import ctypes as ct

import pytest

from paper_2605_30852_amd import binding as B


def cache(**kw):
    d = dict(kv=4096, page_table=8192, lens=12288, refs=16384, n_layers=2, num_pages=10, max_seqs=4, max_pages=5, n_kv_heads=2,
             head_dim=128, dtype=B.SPD_BF16)
    d.update(kw)
    return B.spd_cache(*[d[k] for k, _ in B.spd_cache._fields_])


BIG = 1 << 30


def reserve(c=None, **kw):
    d = dict(seqs=4, add=8, n=2, status=12, workspace=256, ws_bytes=BIG, stream=0)
    d.update(kw)
    B.spd_cache_reserve(c or cache(), **d)


def append(c=None, **kw):
    d = dict(layer=0, k=16, k_stride=256, v=32, v_stride=256, q=48, q_stride=1024, q_out=64, q_out_stride=1024, n_q_heads=8,
             dtype=B.SPD_BF16, rope_cos=80, rope_sin=96, rope_positions=80, seqs=4, cu_rows=8, nseqs=2, rows=3, stream=0)
    d.update(kw)
    B.spd_cache_append(c or cache(), **d)


def prompt(c=None, **kw):
    d = dict(layer=0, q=16, q_stride=1024, out=32, out_stride=1024, n_q_heads=8, dtype=B.SPD_BF16, seqs=4, cu_rows=8, nseqs=2,
             rows=3, max_len=0, workspace=256, ws_bytes=BIG, stream=0)
    d.update(kw)
    B.spd_prompt_attention(c or cache(), **d)


def prefix(c=None, **kw):
    d = dict(layer=0, q=16, q_stride=1024, out=32, out_stride=1024, n_q_heads=8, dtype=B.SPD_BF16, seqs=4, nseqs=2, cu_groups=8,
             prefix_lens=12, ngroups=1, max_len=0, workspace=256, ws_bytes=BIG, stream=0)
    d.update(kw)
    B.spd_prefix_attention(c or cache(), **d)


def refused(call, *a, code=B.SPD_E_INVAL, **kw):
    with pytest.raises(B.SPDError) as e:
        call(*a, **kw)
    assert e.value.status == code
    assert str(e.value).strip()


BAD_CACHES = [dict(kv=0), dict(kv=4104), dict(page_table=0), dict(page_table=8194), dict(lens=0), dict(n_layers=0), dict(num_pages=0),
              dict(max_seqs=0), dict(max_seqs=65537), dict(max_pages=0), dict(max_pages=(1 << 26) + 1), dict(n_kv_heads=0),
              dict(head_dim=96), dict(dtype=2)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_a_bad_cache(bad):
    for call in (reserve, append, prompt, prefix):
        refused(call, cache(**bad))


@pytest.mark.parametrize("bad", [dict(seqs=0), dict(add=0), dict(add=2), dict(status=0), dict(n=0), dict(n=5), dict(workspace=0),
                                 dict(workspace=128)], ids=str)
def test_reserve(bad):
    refused(reserve, **bad)


def test_the_other_page_calls():
    c = cache()
    refused(reserve, cache(refs=0))
    for n in (0, 5):
        refused(B.spd_cache_fork, c, 4, 8, 12, n, 16, 256, BIG, 0)
        refused(B.spd_cache_truncate, c, 4, 8, n, 16, 256, BIG, 0)
        refused(B.spd_cache_workspace, c, n)
    refused(B.spd_cache_fork, c, 4, 0, 12, 2, 16, 256, BIG, 0)
    refused(B.spd_cache_truncate, c, 4, 8, 2, 0, 256, BIG, 0)
    refused(B.spd_cache_compact, c, 0, 256, BIG, 0)
    need = B.spd_cache_workspace(c, 2)
    assert need >= 4 * (4 * 2 + 3 * 10)
    with pytest.raises(B.SPDError) as e:
        reserve(ws_bytes=16)
    assert e.value.status == B.SPD_E_CAPACITY and "bytes needed" in str(e.value)
    refused(B.spd_cache_compact, c, 4, 256, 16, 0, code=B.SPD_E_CAPACITY)


@pytest.mark.parametrize("bad", [
    dict(layer=-1), dict(layer=2), dict(k=0), dict(k=24), dict(k_stride=255), dict(k_stride=264 - 4), dict(k_stride=248), dict(v=0),
    dict(v_stride=128), dict(q=0), dict(q_out=0), dict(n_q_heads=0), dict(q_stride=1016), dict(q_out_stride=1020), dict(dtype=3),
    dict(rope_cos=0), dict(rope_sin=0), dict(rope_cos=84), dict(rope_positions=79), dict(rope_cos=0, rope_sin=0), dict(seqs=0),
    dict(cu_rows=0), dict(cu_rows=9), dict(nseqs=0), dict(nseqs=5), dict(rows=-1)], ids=str)
def test_append(bad):
    refused(append, **bad)


def test_append_of_no_rows_is_nothing():
    append(rows=0)
    append(rows=0, q=0, q_out=0, n_q_heads=0)
    append(rows=0, rope_cos=0, rope_sin=0, rope_positions=0)


@pytest.mark.parametrize("bad", [
    dict(layer=2), dict(q=0), dict(q=24), dict(out=0), dict(q_stride=1023), dict(q_stride=1016), dict(out_stride=1020), dict(n_q_heads=0),
    dict(n_q_heads=7), dict(n_q_heads=34), dict(dtype=2), dict(seqs=0), dict(nseqs=0), dict(nseqs=65537), dict(max_len=-1)], ids=str)
def test_attention(bad):
    refused(prompt, **bad)
    refused(prefix, **bad)


def test_attention_of_one_kind():
    refused(prompt, cu_rows=0)
    refused(prompt, rows=-1)
    prompt(rows=0)
    refused(prefix, ngroups=0)
    refused(prefix, cu_groups=0)
    refused(prefix, prefix_lens=0)
    refused(prefix, ngroups=3)
    refused(prefix, prefix_lens=2)
    refused(prefix, cache(max_seqs=5000), nseqs=4097)
    for call in (prompt, prefix):
        refused(call, cache(dtype=B.SPD_F32))  # bf16 queries over an fp32 cache


def test_null_outputs():
    c = cache()
    assert B.lib().spd_cache_workspace(ct.byref(c), 1, None) == B.SPD_E_INVAL
    assert B.lib().spd_prompt_attention_workspace(ct.byref(c), 8, B.SPD_BF16, 1, 1, 0, None) == B.SPD_E_INVAL
    assert B.lib().spd_prefix_attention_workspace(ct.byref(c), 8, B.SPD_BF16, 1, 0, 0, None) == B.SPD_E_INVAL
    assert B.lib().spd_cache_reserve(None, 4, 8, 1, 12, 256, BIG, 0) == B.SPD_E_INVAL


def test_attention_in_place():
    for call in (prompt, prefix):
        refused(call, q=32, out=32)
