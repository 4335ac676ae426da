"""Free pages and compaction where one workgroup's work ends: 64 sequences, 16384 entries, 32768 pages, and one more of each."""
import numpy as np
import pytest

from oracle import pages as OP
from test_gpu_pages import GUARD, dev, guarded, in_use

pytestmark = pytest.mark.gpu
SHAPES = [(64, 256, 32768), (64, 256, 32767), (64, 256, 32769), (64, 257, 32768), (65, 252, 32768), (1, 16384, 32768), (1, 16385, 32768), (16, 1024, 32768), (63, 260, 32736), (64, 256, 600)]


@pytest.mark.parametrize("wild", [False, True])
@pytest.mark.parametrize("batch, cols, n_pages", SHAPES)
def test_free_and_compacted(batch, cols, n_pages, wild):
    import paper_2602_24174_amd as T
    rng = np.random.default_rng(batch * cols + n_pages + wild)
    table, pages = in_use(rng, batch, cols, n_pages, wild)
    if not wild:
        pages[0] = cols
        table[0, cols - 1] = n_pages - 1                    # the last entry, and the last page
    held = np.clip(pages, 0, cols).tolist()
    free, summary = guarded(n_pages), guarded(3)
    T.tasc_pages_free(dev(table), dev(pages), n_pages, free[:n_pages], summary[:3])
    want = OP.free(table.tolist(), held, n_pages)
    assert (free.tolist(), summary.tolist()) == (want[0] + [-9] * GUARD, want[1] + [-9] * GUARD)
    for cap in (n_pages // 2, 700, 1):
        tab, frm, to, summary = dev(table), guarded(cap), guarded(cap), guarded(3)
        T.tasc_pages_compact(tab, dev(pages), n_pages, tab, frm[:cap], to[:cap], summary[:3])
        after, a, b, s = OP.compact(table.tolist(), held, n_pages, cap)
        assert tab.tolist() == after and summary.tolist() == s + [-9] * GUARD
        assert frm.tolist() == a + [-9] * GUARD and to.tolist() == b + [-9] * GUARD
