"""CPU checks of the paged calls: everything the host can see is refused before the device is touched."""
import ctypes
import os

import pytest

NULL, SHAPE, WS, DTYPE = 1, 2, 5, 7
AT = 0x1000                                                # never followed


@pytest.fixture(scope="module")
def ada():
    from paper_2605_03110_amd import ada as mod
    if not os.path.exists(mod.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return mod


def cache_of(ada, **over):
    d = dict(K=AT, V=AT, bounds=AT, pages=10, page=16, H_kv=2, d_h=64, dtype=ada.ADA_BF16, page_stride=2048, head_stride=1024, slot_stride=64)
    d.update(over)
    return ada.AdaPagedCache(**d)


def chunk_of(ada, **over):
    d = dict(B=2, rows=8, longest=4, max_pages=5, table=AT, table_stride=5, start=AT, past=AT)
    d.update(over)
    return ada.AdaPagedChunk(**d)


def calls(ada, cache, chunk, H=4, status=AT, Q=AT, ldq=256):
    """The status of each of the four calls."""
    L, c, k = ada.lib(), None if cache is None else ctypes.byref(cache), None if chunk is None else ctypes.byref(chunk)
    return (L.ada_cache_append(c, k, Q, ldq, AT, 128, AT, 128, H, None, None, 0.0, None, 0, 0, AT, 256, status, None, 0),
            L.ada_attention_paged(c, k, Q, H, ldq, AT, 256, status, AT, 1 << 40, None, 0),
            L.ada_select_pages(c, k, Q, H, ldq, 3, 1, 1, AT, AT, status, AT, 1 << 40, None, 0),
            L.ada_attention_pages(c, k, Q, H, ldq, AT, AT, 3, AT, 256, status, AT, 1 << 40, None, 0))


@pytest.mark.parametrize("over", [
    dict(page=8), dict(page=48), dict(page=512), dict(pages=0), dict(H_kv=0), dict(d_h=96), dict(d_h=32), dict(slot_stride=63), dict(slot_stride=68),
    dict(head_stride=32), dict(page_stride=-2048), dict(page_stride=2052), dict(K=AT + 8), dict(V=AT + 2), dict(bounds=AT + 4), dict(H_kv=3),
    dict(d_h=256, dtype=0, slot_stride=256)])
def test_caches_that_are_refused(ada, over):
    assert calls(ada, cache_of(ada, **over), chunk_of(ada)) == (SHAPE,) * 4


@pytest.mark.parametrize("over", [
    dict(B=0), dict(B=5000), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(longest=9), dict(longest=0), dict(max_pages=0), dict(table_stride=4),
    dict(max_pages=1 << 23, table_stride=1 << 23)])
def test_chunks_that_are_refused(ada, over):
    assert calls(ada, cache_of(ada), chunk_of(ada, **over)) == (SHAPE,) * 4


def test_missing_pointers_and_types(ada):
    assert calls(ada, None, chunk_of(ada)) == (NULL,) * 4
    assert calls(ada, cache_of(ada), None) == (NULL,) * 4
    for over in (dict(K=None), dict(V=None)):
        assert calls(ada, cache_of(ada, **over), chunk_of(ada)) == (NULL,) * 4
    for over in (dict(table=None), dict(start=None), dict(past=None)):
        assert calls(ada, cache_of(ada), chunk_of(ada, **over)) == (NULL,) * 4
    assert calls(ada, cache_of(ada), chunk_of(ada), status=None) == (NULL,) * 4
    assert calls(ada, cache_of(ada), chunk_of(ada), Q=None) == (NULL,) * 4
    assert calls(ada, cache_of(ada, dtype=9), chunk_of(ada)) == (DTYPE,) * 4
    assert calls(ada, cache_of(ada, bounds=None), chunk_of(ada))[2] == NULL


def test_rows_of_queries(ada):
    assert calls(ada, cache_of(ada), chunk_of(ada), H=3) == (SHAPE,) * 4
    assert calls(ada, cache_of(ada), chunk_of(ada), H=0) == (SHAPE,) * 4
    assert calls(ada, cache_of(ada), chunk_of(ada), ldq=255) == (SHAPE,) * 4
    assert calls(ada, cache_of(ada), chunk_of(ada), ldq=260) == (SHAPE,) * 4
    assert calls(ada, cache_of(ada), chunk_of(ada), Q=AT + 8) == (SHAPE,) * 4


def test_single_arguments(ada):
    L, c, k = ada.lib(), ctypes.byref(cache_of(ada)), ctypes.byref(chunk_of(ada))

    def append(rope=None, rot=0, rope_len=0, eps=0.0, qn=None, ldk=128, ldv=128, out=AT, ldo=256, Q=AT):
        return L.ada_cache_append(c, k, Q, 256, AT, ldk, AT, ldv, 4, qn, None, eps, rope, rot, rope_len, out, ldo, AT, None, 0)
    for bad in (dict(rope=AT, rot=8, rope_len=4), dict(rope=AT, rot=72, rope_len=4), dict(rope=AT, rot=80, rope_len=4), dict(rope=AT, rot=32, rope_len=0),
                dict(rope=AT + 4, rot=32, rope_len=4), dict(qn=AT, eps=-1.0), dict(qn=AT, eps=float("nan")), dict(qn=AT + 2), dict(ldk=64), dict(ldv=132),
                dict(ldo=255), dict(out=AT + 4)):
        assert append(**bad) == SHAPE, bad
    assert append(out=None) == NULL and append(Q=None) == NULL

    def pick(budget=3, first=1, last=1, chunk=k, pages=AT, counts=AT, ws=AT, n=1 << 40):
        return L.ada_select_pages(c, chunk, AT, 4, 256, budget, first, last, pages, counts, AT, ws, n, None, 0)
    assert pick(budget=0) == SHAPE and pick(first=-1) == SHAPE and pick(last=3) == SHAPE and pick(first=2, last=2) == SHAPE
    assert pick(pages=None) == NULL and pick(counts=None) == NULL and pick(ws=None) == NULL
    assert pick(ws=AT + 64) == WS and pick(n=1000) == WS
    assert pick(chunk=ctypes.byref(chunk_of(ada, max_pages=8193, table_stride=8193))) == SHAPE

    def attend(ws=AT, n=1 << 40, out=AT, ldo=256):
        return L.ada_attention_paged(c, k, AT, 4, 256, out, ldo, AT, ws, n, None, 0)
    assert attend(ws=None) == NULL and attend(out=None) == NULL
    assert attend(ws=AT + 128) == WS and attend(n=100) == WS and attend(ldo=248) == SHAPE
    assert L.ada_attention_pages(c, k, AT, 4, 256, None, AT, 3, AT, 256, AT, AT, 1 << 40, None, 0) == NULL
    assert L.ada_attention_pages(c, k, AT, 4, 256, AT, AT, 0, AT, 256, AT, AT, 1 << 40, None, 0) == SHAPE


def test_workspace_size(ada):
    n = ada.lib().ada_paged_workspace_bytes(ctypes.byref(cache_of(ada)), ctypes.byref(chunk_of(ada)), 4)
    assert n > 0 and n % 256 == 0
    assert ada.lib().ada_paged_workspace_bytes(ctypes.byref(cache_of(ada)), ctypes.byref(chunk_of(ada)), 3) == 0
