"""What the serving operators refuse, by their status and before anything is enqueued (no device is needed: the addresses are never
followed)."""
import ctypes as C
import os

import pytest

import paper_2602_24174_amd as T
from paper_2602_24174_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(T.LIB_PATH), reason="libtasc.so is not built")

A = 1 << 20            # an aligned address


def status(name, *args):
    rc = getattr(T.lib(), name)(*args)
    assert rc == 0 or T.lib().tasc_last_error()
    return rc


def test_page_tables():
    good = dict(kv_len=A, new_rows=A, held=A, batch=4, free=A, n_free=8, table=A, max_pages=4, pages=2 * A, row_off=A, slots=A, cap=8, summary=A)

    def call(**kw):
        a = dict(good, **kw)
        return status("tasc_page_tables", *a.values(), None)

    for bad in (dict(kv_len=None), dict(table=None), dict(batch=0), dict(batch=-1), dict(batch=(1 << 20) + 1), dict(max_pages=0), dict(max_pages=1 << 27),
                dict(n_free=-1), dict(n_free=1 << 27), dict(cap=-1), dict(slots=None), dict(pages=A, held=A)):
        assert call(**bad) == B.TASC_EINVAL, bad


def cache(**kw):
    return B.Kv4CacheDesc(**dict(dict(pool=A, n_pages=4, n_kv_heads=2, head_dim=64), **kw))


BAD_CACHES = [dict(pool=None), dict(pool=A + 64), dict(n_pages=0), dict(n_pages=1 << 27), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=16),
              dict(head_dim=96), dict(head_dim=256)]


def test_cache_shapes():
    assert T.tasc_kv4_page_bytes(2, 128) == 2 * 2304 and T.tasc_kv4_page_bytes(3, 64) == 3 * 1152 and T.tasc_kv4_page_bytes(1, 32) == 640
    assert [T.tasc_kv4_page_bytes(*s) for s in ((0, 64), (1025, 64), (2, 48), (2, 256), (2, 0))] == [0] * 5


def test_append_and_read():
    def append(c=None, k=A, v=A, dtype=0, ks=128, vs=128, slots=A, rows=3):
        return status("tasc_kv4_append", C.byref(c or cache()), k, v, dtype, ks, vs, slots, rows, None)

    def read(c=None, slots=A, rows=3, dtype=0, k=A, v=A):
        return status("tasc_kv4_read", C.byref(c or cache()), slots, rows, dtype, k, v, None)

    for bad in BAD_CACHES:
        assert append(cache(**bad)) == B.TASC_EINVAL and read(cache(**bad)) == B.TASC_EINVAL, bad
    for bad in (dict(k=None), dict(v=None), dict(slots=None), dict(dtype=2), dict(dtype=-1), dict(ks=-1), dict(vs=-1), dict(rows=-1), dict(k=A + 2),
                dict(v=A + 1, dtype=1)):
        assert append(**bad) == B.TASC_EINVAL, bad
    for bad in (dict(k=None), dict(v=None), dict(slots=None), dict(dtype=7), dict(rows=-1), dict(k=A + 8)):
        assert read(**bad) == B.TASC_EINVAL, bad
    assert append(rows=0, k=None, v=None, slots=None) == 0 and read(rows=0, k=None, v=None, slots=None) == 0
    assert status("tasc_kv4_append", None, A, A, 0, 1, 1, A, 1, None) == B.TASC_EINVAL


def test_attention():
    good = dict(q=A, out=A, q_stride=256, out_stride=256, table=A, row_off=A, kv_len=A, max_pages=8, batch=2, rows=4, n_heads=4, max_rows=2, max_kv=128, scale=0.1)

    def call(c=None, ws=A, n=1 << 30, **kw):
        return status("tasc_kv4_attention", C.byref(c or cache()), C.byref(B.Kv4Attn(**dict(good, **kw))), ws, n, None)

    for bad in BAD_CACHES:
        assert call(cache(**bad)) == B.TASC_EINVAL, bad
    for bad in (dict(q=None), dict(out=None), dict(table=None), dict(row_off=None), dict(kv_len=None), dict(max_pages=0), dict(batch=-1), dict(rows=-1), dict(n_heads=3),
                dict(n_heads=0), dict(max_rows=-1), dict(max_kv=-1), dict(q=A + 8), dict(out=A + 2), dict(q_stride=260), dict(out_stride=250), dict(out_stride=252),
                dict(q_stride=-256), dict(max_pages=(1 << 27) + 1), dict(max_pages=(1 << 26) + 1), dict(max_rows=1 << 30)):
        assert call(**bad) == B.TASC_EINVAL, bad
    for none in (dict(batch=0), dict(rows=0), dict(max_rows=0)):
        assert call(**none) == 0, none
    need = T.tasc_kv4_attention_workspace_bytes(2, 4, 4, 2, 64, 2, 100000)
    assert need > 0
    assert call(max_kv=100000, n=need - 1) == B.TASC_ENOMEM and call(max_kv=100000, ws=None) == B.TASC_ENOMEM
    assert call(max_kv=100000, ws=A + 4) == B.TASC_EINVAL
    assert status("tasc_kv4_attention", C.byref(cache()), None, A, 1 << 30, None) == B.TASC_EINVAL
    for shape in ((0, 4, 4, 2, 64, 2, 128), (2, 0, 4, 2, 64, 2, 128), (2, 4, 3, 2, 64, 2, 128), (2, 4, 4, 2, 48, 2, 128), (2, 4, 4, 2, 64, 0, 128), (2, 4, 4, 2, 64, 2, -1)):
        assert T.tasc_kv4_attention_workspace_bytes(*shape) == 0


def test_accept_sampled():
    good = dict(logits=A, dtype=0, stride=100, batch=3, k=2, vocab=100, drafts=A, probs=A, temperature=A, u=A, accept_len=A, emitted=A, logprob=A, ws=A, n=1 << 20)

    def call(**kw):
        return status("tasc_accept_sampled", *dict(good, **kw).values(), None)

    for bad in (dict(logits=None), dict(u=None), dict(accept_len=None), dict(emitted=None), dict(drafts=None), dict(dtype=2), dict(stride=99), dict(batch=-1),
                dict(batch=30000), dict(k=-1), dict(k=16), dict(vocab=1), dict(vocab=(1 << 24) + 1, stride=1 << 25), dict(logits=A + 2), dict(ws=A + 8)):
        assert call(**bad) == B.TASC_EINVAL, bad
    need = T.tasc_accept_sampled_workspace_bytes(3, 2, 100)
    assert call(n=need - 1) == B.TASC_ENOMEM and call(ws=None) == B.TASC_ENOMEM
    assert call(batch=0) == 0
    for shape in ((0, 2, 100), (3, -1, 100), (3, 16, 100), (3, 2, 1), (3, 2, (1 << 24) + 1)):
        assert T.tasc_accept_sampled_workspace_bytes(*shape) == 0


def test_host_tensors_are_refused():
    import torch
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(T.TascError):
        T.tasc_page_tables(i, i, i, i, torch.zeros((4, 4), dtype=torch.int32))
    with pytest.raises(T.TascError):
        T.tasc_accept_sampled(torch.zeros((4, 1, 8)), None, None, None, torch.zeros((4, 1, 2)), i, i)
