"""Refusals of the serving operators at the limits of their arguments (no GPU needed).

Every call here fails validation or has nothing to do, which returns before any HIP call is made.
"""
import ctypes

import pytest

import libutil
from paper_2607_23265_amd import serve
from test_serve_capi import ALIGN, AT, NULL, OK, append, cache, ragged, turn


@pytest.fixture(scope="module")
def L():
    libutil.ensure_built()
    return serve.lib()


def test_queries_without_a_token_to_store(L):
    """max_tokens = 0: queries are rotated all the same, so their arguments are looked at."""
    none = ragged(max_tokens=0)
    assert append(L, r=none, q=None) == OK
    assert append(L, r=none, out=None) == NULL and append(L, r=none, out=2 * AT + 8) == ALIGN
    assert append(L, r=none, t=turn(positions=None)) == NULL


def test_structs_are_told_apart_by_more_than_their_size(L):
    """Bytes of a cache's and a batch's size that are neither."""
    from paper_2607_23265_amd import _serve
    for size in (48, 52, 56, 60, 64):
        with pytest.raises(ValueError, match="expected"):
            _serve.workspace(bytes(size), bytes(size), 4, 1, 0)


@pytest.mark.parametrize("kind,fields", [(serve.PagedCache, ("k", "v", "k_scale", "v_scale", "c")),
                                         (serve.Ragged, ("start", "kv_len", "table", "max_tokens", "max_kv", "c")),
                                         (serve.Rotation, ("table", "sections", "interleaved", "c"))])
def test_fields_cannot_be_assigned(kind, fields):
    """An assigned field would leave the packed struct with the old address or value."""
    x = kind.__new__(kind)
    for name in (*fields, "max_pages"):
        with pytest.raises(AttributeError):
            setattr(x, name, 1)


@pytest.mark.parametrize("n,kv,shared", [
    (1286, 1323, False), (1600, 1600, False), (2200, 2200, False), (1000, 5000, False), (100, 1600, False),
    (100, 3100, True), (300, 6300, True), (400, 16400, True)])
def test_prompts_are_shared_where_that_is_faster(L, n, kv, shared):
    """28 query heads of 128 over 4: the measured side of each (a workspace is needed where blocks are shared)."""
    r = ragged(batch=1, tokens=n, max_tokens=n, max_kv=kv, table_stride=kv)
    f = serve._Attention(28, 1, 0, 0.1)
    need = L.wz_attention_workspace_bytes(ctypes.byref(cache()), ctypes.byref(r), ctypes.byref(f))
    assert (need > 0) == shared
