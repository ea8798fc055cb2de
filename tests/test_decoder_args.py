"""Refusals of the decoder's operators, all on the host: the pointers below are
addresses that nothing may touch, so every call has to end in its checks."""
import ctypes

import pytest

from paper_2605_01060_amd import surge as S

A = 1 << 20  # 16-byte aligned addresses
PAGES, TABLE, LENGTHS, X, Y, Q, O, CU = (A + (i << 12) for i in range(8))
NAN, INF = float("nan"), float("inf")
GOOD = dict(pages=PAGES, n_pages=9, page_tokens=32, n_kv_heads=2, d_head=64, table=TABLE, ld_table=4,
            n_seqs=3, lengths=LENGTHS, max_length=128)


def cache(**change):
    return S.KVCache(**{**GOOD, **change})


def refused(fn, args, **change):
    with pytest.raises(S.SurgeError) as e:
        fn(**{**args, **change})
    assert e.value.status in (S.SURGE_ERR_INVALID_ARGUMENT, S.SURGE_ERR_CAPACITY), e.value
    return e.value


STORE = dict(n_rows=6, d_cu=CU, d_k=X, ld_k=128, d_v=Y, ld_v=128)
ATTEND = dict(n_rows=6, d_cu=CU, max_rows=4, n_heads=4, causal=1, scale=0.125, d_q=Q, ld_q=256,
              workspace=None, d_out=O, ld_out=256)
CALLS = [(S.surge_op_cache_write, STORE), (S.surge_op_cache_read, STORE),
         (S.surge_op_cache_attention, ATTEND)]


@pytest.mark.parametrize("change", [
    dict(pages=0), dict(pages=A + 8), dict(n_pages=0), dict(n_pages=1 << 31), dict(page_tokens=8),
    dict(page_tokens=48), dict(page_tokens=512), dict(page_tokens=0), dict(page_tokens=-16),
    dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(d_head=48), dict(d_head=256), dict(d_head=0),
    dict(table=0), dict(table=A + 2), dict(ld_table=3), dict(max_length=129), dict(max_length=-1),
    dict(max_length=(1 << 30) + 1, ld_table=1 << 27), dict(n_seqs=-1), dict(n_seqs=(1 << 20) + 1),
    dict(lengths=0), dict(lengths=A + 1),
])
@pytest.mark.parametrize("fn,args", CALLS)
def test_refused_caches(fn, args, change):
    refused(fn, args, cache=cache(**change))


@pytest.mark.parametrize("change", [
    dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(d_cu=CU + 2), dict(n_rows=7, d_cu=0),
    dict(d_k=0), dict(d_v=0), dict(d_k=X + 8), dict(d_v=Y + 2), dict(ld_k=120), dict(ld_v=132),
    dict(ld_k=(1 << 22) + 8), dict(d_k=PAGES), dict(d_v=PAGES),
])
@pytest.mark.parametrize("fn", [S.surge_op_cache_write, S.surge_op_cache_read])
def test_refused_rows(fn, change):
    refused(fn, STORE, cache=cache(), **change)


def test_read_into_one_matrix_and_too_many_rows():
    refused(S.surge_op_cache_read, STORE, cache=cache(), d_v=X)
    big = cache(n_kv_heads=1024)
    for fn in (S.surge_op_cache_write, S.surge_op_cache_read):
        e = refused(fn, STORE, cache=big, n_rows=1 << 30, ld_k=1024 * 64, ld_v=1024 * 64)
        assert e.status == S.SURGE_ERR_CAPACITY


@pytest.mark.parametrize("change", [
    dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(d_cu=CU + 1), dict(n_rows=7, d_cu=0),
    dict(max_rows=0), dict(max_rows=-1), dict(max_rows=1 << 29), dict(n_rows=15, d_cu=0),
    dict(n_heads=0), dict(n_heads=3), dict(n_heads=2048), dict(n_heads=-2), dict(causal=2),
    dict(causal=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF),
    dict(scale=3e38), dict(d_q=0), dict(d_out=0), dict(d_q=Q + 8), dict(d_out=O + 4), dict(ld_q=248),
    dict(ld_out=260), dict(ld_out=1 << 23), dict(d_out=Q), dict(d_out=PAGES),
])
def test_refused_attention(change):
    refused(S.surge_op_cache_attention, ATTEND, cache=cache(), **change)


VERIFY = dict(n_seqs=3, max_drafts=4, vocab=100, d_n_drafts=A, d_drafts=TABLE, d_p=X, ld_p=100, d_q=Y,
              ld_q=100, d_u=Q, workspace=None, d_tokens=O, d_accepted=CU)


@pytest.mark.parametrize("change", [
    dict(n_seqs=-1), dict(n_seqs=(1 << 20) + 1), dict(max_drafts=-1), dict(max_drafts=1025),
    dict(vocab=0), dict(vocab=(1 << 22) + 1), dict(d_n_drafts=A + 1), dict(d_drafts=0),
    dict(d_drafts=TABLE + 2), dict(d_p=0), dict(d_p=X + 2), dict(ld_p=99), dict(d_q=Y + 1),
    dict(ld_q=99), dict(ld_p=(1 << 30) + 1), dict(d_u=0), dict(d_u=Q + 2), dict(d_tokens=0),
    dict(d_accepted=0), dict(d_tokens=TABLE), dict(d_accepted=A), dict(d_accepted=O), dict(d_tokens=X),
])
def test_refused_verification(change):
    refused(S.surge_op_verify_drafts, VERIFY, **change)


def test_refused_sizes():
    for args in ((8, 1, 64), (32, 0, 64), (32, 1, 96), (512, 1, 64), (32, 1025, 64)):
        with pytest.raises(S.SurgeError):
            S.surge_cache_page_bytes(*args)
    for args in ((-1, 10), (3, 0), (1 << 21, 10), (1, 1 << 23)):
        with pytest.raises(S.SurgeError):
            S.surge_verify_workspace(*args)
    for c, rows, heads in ((cache(d_head=40), 1, 2), (cache(), -1, 2), (cache(), 1, 3), (cache(), 1, 0)):
        with pytest.raises(S.SurgeError):
            S.surge_cache_attention_workspace(c, rows, heads)


def test_null_structs_and_results():
    lib = S.lib()
    bad = S.SURGE_ERR_INVALID_ARGUMENT
    assert lib.surge_op_cache_write(None, 1, None, X, 64, Y, 64, None) == bad
    assert lib.surge_op_cache_read(None, 1, None, X, 64, Y, 64, None) == bad
    assert lib.surge_op_cache_attention(None, 1, None, 1, 1, 1, 1.0, Q, 64, None, 0, O, 64, None) == bad
    assert lib.surge_cache_attention_workspace(None, 1, 1, ctypes.byref(ctypes.c_int64())) == bad
    assert lib.surge_cache_attention_workspace(ctypes.byref(cache()), 1, 2, None) == bad
    assert lib.surge_cache_page_bytes(32, 1, 64, None) == bad
    assert lib.surge_verify_workspace(1, 1, None) == bad


@pytest.mark.parametrize("page,heads,dh", [(16, 1, 32), (32, 12, 64), (256, 8, 128), (64, 3, 128)])
def test_page_bytes(page, heads, dh):
    """Two rows of codes and two of scales for every position and head."""
    assert S.surge_cache_page_bytes(page, heads, dh) == heads * page * 2 * (dh // 2 + dh // 32)


def test_no_rows_or_sequences_is_a_call_that_does_nothing():
    for c, n in ((cache(), 0), (cache(n_seqs=0), 6)):
        for fn, args in CALLS:
            fn(**{**args, "cache": c, "n_rows": n})
    S.surge_op_verify_drafts(**{**VERIFY, "n_seqs": 0})
    assert S.surge_cache_attention_workspace(cache(n_seqs=0), 4, 4) == 0
    assert S.surge_cache_attention_workspace(cache(), 0, 4) == 0


@pytest.mark.parametrize("max_rows", [1 << 62, (1 << 62) + 1, (1 << 63) - 1, 1 << 54, (1 << 28) + 1])
def test_refused_max_rows_whose_product_with_the_heads_wraps(max_rows):
    """2^62 rows of 4 heads are 2^64, 0 in 64 bits."""
    refused(S.surge_op_cache_attention, ATTEND, cache=cache(), max_rows=max_rows)
    with pytest.raises(S.SurgeError):
        S.surge_cache_attention_workspace(cache(), max_rows, 4)
