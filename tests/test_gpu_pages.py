"""Pages that are forked, copied, freed and moved, against their oracle: every output equal, and what must stay as it was untouched."""
import numpy as np
import pytest

from oracle import pages as OP

pytestmark = pytest.mark.gpu
GUARD = 5


def dev(x):
    import torch
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def guarded(n):
    import torch
    return torch.full((n + GUARD,), -9, dtype=torch.int32, device="cuda")


def fork(src, dst, new, kv_len, table, pages, summary=True):
    import paper_2602_24174_amd as T
    n = len(src)
    kv, tab, pg, frm, to, s = dev(kv_len), dev(table), dev(pages), guarded(n), guarded(n), guarded(3)
    T.tasc_pages_fork(dev(src), dev(dst), kv, tab, pg, None if new is None else dev(new), frm[:n], to[:n], s[:3] if summary else None)
    assert (frm[n:] == -9).all() and (to[n:] == -9).all() and (s[3:] == -9).all()
    got = kv.tolist(), tab.tolist(), pg.tolist(), frm[:n].tolist(), to[:n].tolist()
    want_kv, want_table, want_pages = list(kv_len), [list(r) for r in table], list(pages)
    want = OP.fork(list(src), list(dst), new, want_kv, want_table, want_pages)
    assert got == (want_kv, want_table, want_pages, want[0], want[1])
    assert s[:3].tolist() == (want[2] if summary else [-9] * 3)


@pytest.mark.parametrize("batch, cols, n", [(2, 1, 1), (9, 7, 8), (64, 40, 50), (300, 600, 299), (1000, 5, 700)])
def test_forks(batch, cols, n):
    rng = np.random.default_rng(batch)
    kv = rng.integers(0, 16 * cols + 1, batch)
    pages = np.minimum(-(-kv // 16) + rng.integers(0, 2, batch), cols)
    table = rng.permutation(batch * cols).reshape(batch, cols)
    at = rng.permutation(batch)
    sources = at[:max(1, batch - n)]
    dst = at[len(sources):][:n]
    src = rng.choice(sources, len(dst))
    fork(src.tolist(), dst.tolist(), (batch * cols + np.arange(len(dst))).tolist(), kv.tolist(), table.tolist(), pages.tolist(), summary=batch != 9)


def test_forks_that_are_refused():
    kv, pages = [20, 20, -1, 33, 5, 0, 32, 17, 40, 2147483647], [2, 1, 1, 4, 1, 0, 2, 2, 3, 3]
    table = [[10 * b + c for c in range(3)] for b in range(10)]
    #         ok one range range two <0 beyond no   page  len  again   continued
    src = [0, 0, 0, -1, 1, 2, 3, 0, 9, 0, 6]
    dst = [4, 0, 10, 1, 5, 5, 5, 4, 5, 7, 8]
    new = [100, 101, 102, 103, 104, 105, 106, 107, 108, -1, -1]
    fork(src, dst, new, kv, table, pages)
    fork([0, 1, 6], [1, 2, 3], [9, 8, 7], kv, table, [2] * 10)
    fork([0, 6], [1, 2], None, kv, table, [2] * 10)
    fork([0, 7], [1, 2], [1 << 27, (1 << 27) - 1], kv, table, [2] * 10)
    rng = np.random.default_rng(1)
    for _ in range(5):                                     # everything at once
        n = 400
        fork(rng.integers(-1, 11, n).tolist(), rng.integers(-1, 11, n).tolist(), rng.integers(-1, 50, n).tolist(), rng.integers(-3, 60, 10).tolist(), table,
             rng.integers(0, 5, 10).tolist())


def test_no_forks():
    fork([], [], [], [3, 4], [[1], [2]], [1, 1])
    fork([], [], None, [3, 4], [[1], [2]], [1, 1], summary=False)


@pytest.mark.parametrize("page, n_pages, layers, n", [(16, 9, 1, 3), (640, 50, 3, 20), (1152, 40, 2, 20), (4608, 300, 5, 140), (8192, 20, 2, 9), (8208, 20, 2, 10), (18432, 64, 4, 30),
                                                      (131072 + 16, 6, 2, 3)])
def test_copies(page, n_pages, layers, n):
    import torch
    import paper_2602_24174_amd as T
    rng = np.random.default_rng(page)
    stride = n_pages * page + (48 if layers > 2 else 0)
    pool = torch.randint(0, 256, (layers * stride + 64,), dtype=torch.uint8, device="cuda")
    order = rng.permutation(n_pages)
    to, frm = order[:n], rng.choice(order[n:], n)
    frm[n // 3], to[n // 2] = -1, n_pages                   # pairs that copy nothing
    frm[-1] = to[-1]
    want = pool.clone()
    for a, b in zip(frm.tolist(), to.tolist()):
        if 0 <= a < n_pages and 0 <= b < n_pages:
            for j in range(layers):
                want[j * stride + b * page:j * stride + (b + 1) * page] = pool[j * stride + a * page:j * stride + (a + 1) * page]
    T.tasc_pages_copy(pool, page, n_pages, layers, dev(frm), dev(to), layer_stride=stride)
    assert torch.equal(pool, want)


def test_copies_beyond_32_bits():
    import torch
    import paper_2602_24174_amd as T
    page, n_pages, layers = 1 << 16, 70000, 2               # 4.6 GB a layer
    pool = torch.zeros((layers, n_pages, page), dtype=torch.uint8, device="cuda")
    pool[:, 69999] = 7
    pool[0, 3], pool[1, 3] = 5, 6
    T.tasc_pages_copy(pool, page, n_pages, layers, dev([69999, 3]), dev([1, 69000]))
    assert (pool[:, 1] == 7).all() and (pool[0, 69000] == 5).all() and (pool[1, 69000] == 6).all()
    assert int(pool[:, 2].max()) == 0 and int(pool[:, 68999].max()) == 0 and int(pool[:, 69001].max()) == 0


def in_use(rng, batch, cols, n_pages, wild=False):
    table = rng.integers(0, n_pages, (batch, cols))
    if wild:
        table[rng.random((batch, cols)) < 0.1] = -1
        table[rng.random((batch, cols)) < 0.1] = n_pages
        table[rng.random((batch, cols)) < 0.02] = 2147483647
        table[rng.random((batch, cols)) < 0.02] = -2147483648
    pages = rng.integers(0, cols + 1, batch)
    if wild:
        pages[rng.random(batch) < 0.1] = -3
        pages[rng.random(batch) < 0.1] = cols + 9
    return table, pages


SHAPES = [(1, 1, 1), (1, 3, 1), (3, 4, 31), (3, 4, 32), (2, 9, 33), (16, 40, 2000), (64, 144, 60000), (64, 1024, 65536), (65, 30, 1500), (64, 2, 65537), (300, 100, 40000),
          (5, 5000, 32768), (7, 9000, 100000), (513, 70, 1 << 17)]


@pytest.mark.parametrize("wild", [False, True])
@pytest.mark.parametrize("batch, cols, n_pages", SHAPES)
def test_free_pages(batch, cols, n_pages, wild):
    import paper_2602_24174_amd as T
    rng = np.random.default_rng(batch * cols + wild)
    table, pages = in_use(rng, batch, cols, n_pages, wild)
    free, summary = guarded(n_pages), guarded(3)
    T.tasc_pages_free(dev(table), dev(pages), n_pages, free[:n_pages], summary[:3])
    want = OP.free(table.tolist(), np.clip(pages, 0, cols).tolist(), n_pages)
    assert (free[n_pages:] == -9).all() and (summary[3:] == -9).all()
    assert (free[:n_pages].tolist(), summary[:3].tolist()) == want
    again = guarded(n_pages)
    T.tasc_pages_free(dev(table), dev(pages), n_pages, again[:n_pages])
    assert (again == free).all()


@pytest.mark.parametrize("wild", [False, True])
@pytest.mark.parametrize("batch, cols, n_pages", SHAPES)
def test_compacted(batch, cols, n_pages, wild):
    import paper_2602_24174_amd as T
    rng = np.random.default_rng(batch * cols + wild + 7)
    table, pages = in_use(rng, batch, cols, n_pages, wild)
    if batch == 64:
        pages[5:] = 0                                       # most requests have ended: pages far from the front
    for cap in (n_pages // 2 + 1, n_pages // 5, 0, 1):
        for in_place in (False, True):
            tab = dev(table)
            out = tab if in_place else tab * 0 - 5
            frm, to, summary = guarded(cap), guarded(cap), guarded(3)
            T.tasc_pages_compact(tab, dev(pages), n_pages, out, frm[:cap], to[:cap], summary[:3] if cap != 1 else None)
            after, a, b, want = OP.compact(table.tolist(), np.clip(pages, 0, cols).tolist(), n_pages, cap)
            if not in_place:
                after = [row[:k] + [-5] * (cols - k) for row, k in zip(after, np.clip(pages, 0, cols).tolist())]
                assert (tab == dev(table)).all()
            assert out.tolist() == after
            assert frm.tolist() == a + [-9] * GUARD and to.tolist() == b + [-9] * GUARD
            assert summary.tolist() == (want if cap != 1 else [-9] * 3) + [-9] * GUARD


def test_full_and_empty_pools():
    import paper_2602_24174_amd as T
    for n in (32, 64, 40, 32768, 65536, 65568):
        for used in (n, 0, n - 1):
            table = np.random.default_rng(n).permutation(n)[None, :].copy()
            free, summary, frm, to = guarded(n), guarded(3), guarded(4), guarded(4)
            T.tasc_pages_free(dev(table), dev([used]), n, free[:n], summary[:3])
            assert (free[:n].tolist(), summary[:3].tolist()) == OP.free(table.tolist(), [used], n)
            out = dev(table)
            T.tasc_pages_compact(dev(table), dev([used]), n, out, frm[:4], to[:4], summary[:3])
            want = OP.compact(table.tolist(), [used], n, 4)
            assert (out.tolist(), frm[:4].tolist(), to[:4].tolist(), summary[:3].tolist()) == want


def test_the_largest_pool():
    """2^27 - 1 pages, a few of them listed, the last among them."""
    import torch
    import paper_2602_24174_amd as T
    n = (1 << 27) - 1
    table = dev([[n - 1, 5, 70000, n, -1, 1 << 20], [5, 2, 99999999, 0, 0, 0]])
    free, summary = torch.empty(n, dtype=torch.int32, device="cuda"), guarded(3)
    T.tasc_pages_free(table, dev([6, 3]), n, free, summary[:3])
    assert summary[:3].tolist() == [n - 6, 6, 7]
    gone = dev([2, 5, 70000, 1 << 20, 99999999, n - 1]).long()
    assert (free[n - 6:] == -1).all() and not torch.isin(gone, free[:n - 6].long()).any()
    assert (free[1:n - 6] > free[:n - 7]).all() and int(free[0]) == 0 and int(free[n - 7]) == n - 2
    out, frm, to = table.clone(), guarded(6), guarded(6)
    T.tasc_pages_compact(table, dev([6, 3]), n, out, frm[:6], to[:6], summary[:3])
    assert frm[:6].tolist() == [n - 1, 99999999, 1 << 20, 70000, -1, -1] and to[:6].tolist() == [0, 1, 3, 4, -1, -1]
    assert out.tolist() == [[0, 5, 4, n, -1, 3], [5, 2, 1, 0, 0, 0]] and summary[:3].tolist() == [6, 4, 6]


def test_replayed_and_on_another_stream():
    import torch
    import paper_2602_24174_amd as T
    rng = np.random.default_rng(5)
    for batch, cols, n_pages in ((8, 20, 400), (100, 40, 9000)):
        states = [in_use(rng, batch, cols, n_pages) for _ in range(4)]
        table, pages, out = dev(states[0][0]), dev(states[0][1]), dev(states[0][0])
        free, summary, cap = guarded(n_pages), guarded(3), n_pages // 2
        frm, to, moved = guarded(cap), guarded(cap), guarded(3)
        ws = [torch.empty(T.tasc_pages_workspace_bytes(n_pages), dtype=torch.uint8, device="cuda") for _ in range(2)]

        def step():
            T.tasc_pages_free(table, pages, n_pages, free[:n_pages], summary[:3], ws[0])
            T.tasc_pages_compact(table, pages, n_pages, out, frm[:cap], to[:cap], moved[:3], ws[1])

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for state in states * 2:
            table.copy_(dev(state[0]))
            pages.copy_(dev(state[1]))
            graph.replay()
            torch.cuda.synchronize()
            tab, pg = state[0].tolist(), state[1].tolist()
            assert (free[:n_pages].tolist(), summary[:3].tolist()) == OP.free(tab, pg, n_pages)
            want = OP.compact(tab, pg, n_pages, cap)
            assert [r[:k] for r, k in zip(out.tolist(), pg)] == [r[:k] for r, k in zip(want[0], pg)]
            assert (frm[:cap].tolist(), to[:cap].tolist(), moved[:3].tolist()) == want[1:]
