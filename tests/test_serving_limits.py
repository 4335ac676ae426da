"""Sizes that no launch holds are refused by name, before anything is enqueued (no device is needed: the addresses are never followed)."""
import ctypes as C
import os

import pytest

import paper_2602_24174_amd as T
from paper_2602_24174_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(T.LIB_PATH), reason="libtasc.so is not built")

A = 1 << 20            # an aligned address
MOST = 2 ** 31 - 1


def refused(name, *args):
    rc = getattr(T.lib(), name)(*args)
    return rc == B.TASC_EINVAL and T.lib().tasc_last_error().decode().startswith(name[5:])


def cache(heads, hd):
    return B.Kv4CacheDesc(A, 4, heads, hd)


def test_rows_of_a_call():
    # 1024 x 128 channels: 2^31 - 1 rows are 2^37 workgroups, of which 32 bits keep none at all
    for heads, hd, rows in ((1024, 128, MOST), (1024, 128, 1 << 18), (8, 128, 1 << 25), (1, 32, 1 << 30)):
        if rows * heads * hd >= 1 << 35:
            assert refused("tasc_kv4_append", C.byref(cache(heads, hd)), A, A, 1, 0, 0, A, rows, None), (heads, hd, rows)
            assert refused("tasc_kv4_read", C.byref(cache(heads, hd)), A, rows, 1, A, A, None), (heads, hd, rows)


def test_pairs_of_a_call():
    def call(batch, max_rows, heads, kv_heads):
        a = B.Kv4Attn(A, A, heads * 128, heads * 128, A, A, A, 8, batch, 64, heads, max_rows, 128, 0.1)
        return refused("tasc_kv4_attention", C.byref(cache(kv_heads, 128)), C.byref(a), A, 1 << 40, None)

    # (65535 sequences of 2^15 rows of a head are 2^31 - 2^15 rows, which a launch holds)
    for shape in ((4096, 16384, 32, 8), (65535, (1 << 15) + 1, 1, 1), (1 << 15, (1 << 24) + 1, 2, 2), (64, 1 << 24, 32, 1)):
        assert call(*shape), shape


def test_arrays_of_page_tables_that_overlap():
    """What is written may lie on nothing else that the call names: every pair of arrays, by its first and by its last element."""
    sizes = dict(kv_len=64, new_rows=64, held=64, batch=None, free=40, n_free=None, table=64 * 7, max_pages=None, pages=64, row_off=65, slots=100, cap=None, summary=3)
    numbers = dict(batch=64, n_free=40, max_pages=7, cap=100)
    read, written = ("kv_len", "new_rows", "held", "free"), ("table", "pages", "row_off", "slots", "summary")
    place = {name: A + 8192 * i for i, name in enumerate(sizes)}

    def call(**kw):
        a = {name: kw.get(name, numbers.get(name, place[name])) for name in sizes}
        return refused("tasc_page_tables", *a.values(), None)

    for w in written:
        for other in read + written:
            if other != w:
                for at in (place[other], place[other] + 4 * (sizes[other] - 1), place[other] - 4 * (sizes[w] - 1)):
                    assert call(**{w: at}), (w, other)
    # the other refusals, with arrays that are apart
    for bad in (dict(kv_len=None), dict(table=None), dict(batch=0), dict(max_pages=0), dict(max_pages=1 << 27), dict(n_free=-1), dict(n_free=1 << 27), dict(cap=-1), dict(slots=None)):
        assert call(**bad), bad
