"""What the operators on pages refuse, by their status and before anything is enqueued (no device is needed: the addresses are never followed)."""
import os

import pytest

import paper_2602_24174_amd as T
from paper_2602_24174_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(T.LIB_PATH), reason="libtasc.so is not built")

A = 1 << 24            # addresses far apart


def status(name, *args):
    rc = getattr(T.lib(), name)(*args)
    assert rc == 0 or T.lib().tasc_last_error()
    return rc


def test_fork():
    good = dict(src=A, dst=2 * A, n=4, new=3 * A, kv=4 * A, table=5 * A, pages=6 * A, batch=8, cols=4, frm=7 * A, to=8 * A, summary=9 * A)

    def call(**kw):
        return status("tasc_pages_fork", *dict(good, **kw).values(), None)

    for bad in (dict(src=None), dict(dst=None), dict(kv=None), dict(table=None), dict(pages=None), dict(frm=None), dict(to=None), dict(n=-1), dict(n=(1 << 14) + 1), dict(batch=0),
                dict(batch=(1 << 20) + 1), dict(cols=0), dict(cols=1 << 27), dict(frm=A), dict(to=7 * A + 4), dict(kv=2 * A), dict(table=6 * A - 8), dict(summary=3 * A)):
        assert call(**bad) == B.TASC_EINVAL, bad
    assert call(n=0, src=None, dst=None, frm=None, to=None, summary=None) == 0


def test_copy():
    good = dict(pool=A, page=640, n_pages=10, layers=3, stride=6400, frm=2 * A, to=3 * A, n=5)

    def call(**kw):
        return status("tasc_pages_copy", *dict(good, **kw).values(), None)

    for bad in (dict(pool=None), dict(pool=A + 8), dict(page=0), dict(page=24), dict(page=(1 << 30) + 16), dict(n_pages=0), dict(n_pages=1 << 27), dict(layers=-1), dict(stride=6384),
                dict(stride=6408), dict(frm=None), dict(to=None), dict(n=-1)):
        assert call(**bad) == B.TASC_EINVAL, bad
    assert call(n=0, frm=None, to=None) == 0 and call(layers=0) == 0


def test_free_and_compact():
    n = 1000
    need = T.tasc_pages_workspace_bytes(n)
    assert need > 0 and T.tasc_pages_workspace_bytes(0) == 0 and T.tasc_pages_workspace_bytes(1 << 27) == 0 and T.tasc_pages_workspace_bytes((1 << 27) - 1) > 0
    head = dict(table=A, pages=2 * A, batch=8, cols=4, n_pages=n)
    frees = dict(head, free=3 * A, summary=4 * A, ws=5 * A, size=need)
    moves = dict(head, out=3 * A, frm=4 * A, to=6 * A, cap=100, summary=7 * A, ws=5 * A, size=need)

    def call(name, good, **kw):
        return status(name, *dict(good, **kw).values(), None)

    for name, good in (("tasc_pages_free", frees), ("tasc_pages_compact", moves)):
        for bad in (dict(table=None), dict(pages=None), dict(batch=0), dict(batch=(1 << 20) + 1), dict(cols=0), dict(cols=1 << 27), dict(n_pages=0), dict(n_pages=1 << 27),
                    dict(ws=5 * A + 8), dict(ws=A), dict(summary=2 * A)):
            assert call(name, good, **bad) == B.TASC_EINVAL, (name, bad)
        assert call(name, good, ws=None) == B.TASC_ENOMEM and call(name, good, size=need - 1) == B.TASC_ENOMEM
    for bad in (dict(free=None), dict(free=A), dict(free=4 * A)):
        assert call("tasc_pages_free", frees, **bad) == B.TASC_EINVAL, bad
    for bad in (dict(out=None), dict(frm=None), dict(to=None), dict(cap=-1), dict(cap=1 << 27), dict(out=A + 16), dict(frm=3 * A), dict(to=4 * A), dict(out=2 * A)):
        assert call("tasc_pages_compact", moves, **bad) == B.TASC_EINVAL, bad


def test_host_tensors_are_refused():
    import torch
    i = torch.zeros(4, dtype=torch.int32)
    t = torch.zeros((4, 4), dtype=torch.int32)
    for call in (lambda: T.tasc_pages_fork(i, i, i, t, i, i, i, i), lambda: T.tasc_pages_copy(torch.zeros(64, dtype=torch.uint8), 16, 2, 1, i, i),
                 lambda: T.tasc_pages_free(t, i, 4, i), lambda: T.tasc_pages_compact(t, i, 4, t, i, i)):
        with pytest.raises(T.TascError):
            call()
