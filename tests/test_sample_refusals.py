"""What the filtered sampling refuses, by its status and before anything is enqueued (no device is needed: the addresses are never followed)."""
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


def test_sample():
    need = T.tasc_sample_workspace_bytes(3, 5000)
    good = dict(logits=A, dtype=0, stride=5000, rows=3, vocab=5000, t=2 * A, k=3 * A, p=4 * A, m=5 * A, u=6 * A, token=7 * A, logprob=8 * A, kept=9 * A, ws=10 * A, n=need)

    def call(**kw):
        return status("tasc_sample", *dict(good, **kw).values(), None)

    for bad in (dict(logits=None), dict(u=None), dict(token=None), dict(dtype=2), dict(dtype=-1), dict(stride=4999), dict(rows=-1), dict(rows=65536), dict(vocab=1), dict(vocab=(1 << 24) + 1, stride=1 << 25),
                dict(logits=A + 2), dict(logits=A + 1, dtype=1), dict(ws=10 * A + 8)):
        assert call(**bad) == B.TASC_EINVAL, bad
    assert call(n=need - 1) == B.TASC_ENOMEM and call(ws=None) == B.TASC_ENOMEM
    assert T.tasc_sample_workspace_bytes(3, 1280) == 0 and call(vocab=1280, ws=None, n=0, dtype=7) == B.TASC_EINVAL
    assert call(rows=0, logits=None, u=None, token=None) == 0
    assert [T.tasc_sample_workspace_bytes(*s) for s in ((0, 100), (65536, 100), (3, 1), (3, (1 << 24) + 1))] == [0] * 4


@pytest.mark.parametrize("vocab", [1281, 4097, 49152, 151936, 1 << 24])
def test_a_workspace_for_more_rows_serves_fewer(vocab):
    sizes = [T.tasc_sample_workspace_bytes(rows, vocab) for rows in list(range(1, 1400)) + [2049, 4096, 65535]]
    assert sizes == sorted(sizes)


def test_filter_logits():
    need = T.tasc_sample_workspace_bytes(9, 5000)
    good = dict(logits=A, dtype=1, stride=5000, batch=3, k=2, vocab=5000, t=2 * A, tk=3 * A, p=4 * A, m=5 * A, out=6 * A, out_stride=5000, kept=9 * A, ws=10 * A, n=need)

    def call(**kw):
        return status("tasc_filter_logits", *dict(good, **kw).values(), None)

    for bad in (dict(logits=None), dict(out=None), dict(dtype=3), dict(stride=4999), dict(out_stride=4999), dict(batch=-1), dict(batch=30000), dict(k=-1), dict(k=16), dict(vocab=1),
                dict(vocab=(1 << 24) + 1, stride=1 << 25, out_stride=1 << 25), dict(out=6 * A + 1), dict(out=A + 2), dict(out=A, out_stride=5008), dict(out=A + 80000), dict(out=A - 80000),
                dict(ws=10 * A + 4)):
        assert call(**bad) == B.TASC_EINVAL, bad
    assert call(n=need - 1) == B.TASC_ENOMEM and call(ws=None) == B.TASC_ENOMEM
    assert call(batch=0, logits=None, out=None) == 0


def test_session_filter():
    assert status("tasc_session_filter", None, A, A, A, A, 1 << 20) == B.TASC_EINVAL


def test_host_tensors_are_refused():
    import torch
    i, f = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    for call in (lambda: T.tasc_sample(torch.zeros((4, 8)), f, i), lambda: T.tasc_filter_logits(torch.zeros((4, 1, 8)), torch.zeros((4, 1, 8)))):
        with pytest.raises(T.TascError):
            call()


def test_arrays_that_overlap():
    need = T.tasc_sample_workspace_bytes(3, 5000)
    sample = dict(logits=A, dtype=0, stride=5000, rows=3, vocab=5000, t=2 * A, k=3 * A, p=4 * A, m=5 * A, u=6 * A, token=7 * A, logprob=8 * A, kept=9 * A, ws=10 * A, n=need)
    masks = dict(logits=A, dtype=0, stride=5000, batch=3, k=0, vocab=5000, t=2 * A, tk=3 * A, p=4 * A, m=5 * A, out=6 * A, out_stride=5000, kept=9 * A, ws=10 * A, n=need)
    rows = 4 * 15000                                        # bytes of the logits
    for name, good, written, read in (("tasc_sample", sample, ("token", "logprob", "kept"), ("t", "k", "p", "m", "u")), ("tasc_filter_logits", masks, ("kept",), ("t", "tk", "p", "m"))):
        bad = [{w: good[r] + 4} for w in written for r in read] + [{w: good[r] - 8} for w in written for r in read]         # (all of it over all of the other is not refused)
        bad += [{w: good["ws"] + need - 4} for w in written] + [{w: A + rows - 4} for w in written] + [{r: good["ws"] + 64} for r in read]
        bad += [{w: good[v] + 8} for w in written for v in written if v != w] + [{w: good[v]} for w in written for v in written if v != w]
        bad += [{"ws": A + 16}, {"ws": A}, {"logits": good["ws"] + need - 16}]
        if "out" in good:
            bad += [{"out": good["ws"] + 4096}, {"out": good["ws"] - rows + 4}, {"kept": 6 * A + rows - 4}, {"tk": 6 * A}, {"out": A, "ws": A + 32}, {"out": A, "kept": A + 8}]
        for kw in bad:
            assert status(name, *dict(good, **kw).values(), None) == B.TASC_EINVAL, (name, kw)
    masks.update(k=1, batch=2, kept=3 * A, n=T.tasc_sample_workspace_bytes(4, 5000))        # a count a row over a top-k a sequence
    assert status("tasc_filter_logits", *masks.values(), None) == B.TASC_EINVAL
