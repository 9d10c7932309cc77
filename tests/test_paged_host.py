"""Refusals of the paged cache's calls: every one comes from the host's checks, before anything is enqueued.  No GPU needed."""
import ctypes as C

import pytest

import paper_2510_11958_amd as pkg
from paper_2510_11958_amd.binding import _PagedCache, _PagePool

P = 1 << 20      # an address that is never read: all calls here are refused


def pool(**kw):
    a = dict(n_pages=8, page_size=16, n_req=2, max_pages=4, block_table=P, held=P, free_pages=P, n_free=P)
    a.update(kw)
    return _PagePool(*a.values())


def cache(**kw):
    a = dict(k=P, v=P, page_stride=0, block_table=P, n_pages=8, page_size=16, n_req=2, max_pages=4, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=1, max_rows=8)
    a.update(kw)
    return _PagedCache(*a.values())


def refused(rc, word, code=pkg.DMTD_EINVAL):
    assert rc == code
    assert word in pkg.load_library().dmtd_last_error(None).decode()


TABLES = dict(start=P, rows=P, max_rows=8, cu=P, pos=P, slots=P, status=P)


@pytest.mark.parametrize("in_pool, args, word", [
    (dict(page_size=8), {}, "page_size"), (dict(page_size=48), {}, "page_size"), (dict(page_size=512), {}, "page_size"),
    (dict(n_req=0), {}, "n_req"), (dict(n_req=8193), {}, "n_req"), (dict(n_pages=0), {}, "n_pages"), (dict(max_pages=0), {}, "max_pages"),
    (dict(max_pages=(1 << 26) + 1), {}, "max_pages"), (dict(block_table=None), {}, "null"), (dict(held=None), {}, "null"), (dict(free_pages=None), {}, "null"),
    (dict(n_free=None), {}, "null"), (dict(held=P + 2), {}, "aligned"), ({}, dict(start=None), "null"), ({}, dict(status=None), "null"), ({}, dict(slots=P + 4), "slots"),
    ({}, dict(cu=P + 1), "aligned"), ({}, dict(max_rows=0), "max_rows"), ({}, dict(max_rows=(1 << 24) + 1), "max_rows"),
])
def test_page_tables_refuses(in_pool, args, word):
    a = dict(TABLES, **args)
    refused(pkg.load_library().dmtd_page_tables(C.byref(pool(**in_pool)), *a.values(), None), word)


BAD_CACHE = [
    (dict(dtype=2), "dtype"), (dict(head_dim=96), "head_dim"), (dict(n_q_heads=5), "n_q_heads"), (dict(n_q_heads=0), "n_q_heads"), (dict(n_q_heads=34), "n_q_heads"),
    (dict(n_kv_heads=0), "n_q_heads"), (dict(max_rows=0), "max_rows"), (dict(max_rows=1 << 25), "max_rows"), (dict(k=None), "null"), (dict(v=None), "null"),
    (dict(block_table=None), "null"), (dict(k=P + 8), "aligned"), (dict(v=P + 2), "aligned"), (dict(page_stride=2 * 16 * 64 - 8), "page_stride"),
    (dict(page_stride=2 * 16 * 64 + 4), "page_stride"), (dict(page_stride=-8), "page_stride"), (dict(page_size=17), "page_size"), (dict(n_req=0), "n_req"),
]
APPEND = dict(qkv=P, ld=512, cu=P, pos=P, slots=P, gain=P, eps=1e-6, rope=P, rope_len=64)
BAD_APPEND = [
    (dict(qkv=None), "qkv"), (dict(qkv=P + 4), "qkv"), (dict(ld=508), "ld"), (dict(ld=514), "ld"), (dict(gain=P + 8), "gain"), (dict(eps=-1.0), "eps"),
    (dict(eps=float("nan")), "eps"), (dict(rope=P + 8), "rotary"), (dict(rope_len=0), "rotary"), (dict(cu=None), "row map"), (dict(pos=None), "row map"), (dict(slots=P + 4), "row map"),
]
ATTENTION = dict(qkv=P, ld=256, start=P, cu=P, max_new=0, gain=P, eps=1e-6, rope=P, rope_len=64, out=P, ldo=256, ws=P, ws_bytes=1 << 40)
BAD_ATTENTION = [
    (dict(qkv=None), "qkv"), (dict(ld=252), "ld"), (dict(start=None), "length"), (dict(cu=P + 2), "length"), (dict(max_new=-1), "max_new"), (dict(max_new=9), "max_new"),
    (dict(out=None), "out"), (dict(out=P + 8), "out"), (dict(ldo=248), "ldo"), (dict(ldo=260), "ldo"), (dict(ws=None), "workspace"), (dict(ws=P + 128), "workspace"),
]


@pytest.mark.parametrize("in_cache, word", BAD_CACHE)
def test_a_bad_cache_is_refused(in_cache, word):
    lib, c = pkg.load_library(), cache(**in_cache)
    refused(lib.dmtd_paged_append(C.byref(c), *APPEND.values(), None), word)
    refused(lib.dmtd_paged_attention(C.byref(c), *ATTENTION.values(), None), word)
    assert lib.dmtd_paged_workspace_bytes(C.byref(c)) == 0


@pytest.mark.parametrize("args, word", BAD_APPEND)
def test_paged_append_refuses(args, word):
    refused(pkg.load_library().dmtd_paged_append(C.byref(cache()), *dict(APPEND, **args).values(), None), word)


@pytest.mark.parametrize("args, word", BAD_ATTENTION)
def test_paged_attention_refuses(args, word):
    refused(pkg.load_library().dmtd_paged_attention(C.byref(cache()), *dict(ATTENTION, **args).values(), None), word)


def test_small_workspace_and_null_structs():
    lib, c = pkg.load_library(), cache()
    need = lib.dmtd_paged_workspace_bytes(C.byref(c))
    assert need > 0
    refused(lib.dmtd_paged_attention(C.byref(c), *dict(ATTENTION, ws_bytes=need - 1).values(), None), "workspace", pkg.DMTD_ECAPACITY)
    refused(lib.dmtd_paged_append(None, *APPEND.values(), None), "null")
    refused(lib.dmtd_paged_attention(None, *ATTENTION.values(), None), "null")
    refused(lib.dmtd_page_tables(None, *TABLES.values(), None), "null")
    assert lib.dmtd_paged_workspace_bytes(None) == 0
