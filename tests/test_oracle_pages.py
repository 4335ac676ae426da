"""Pins of the oracle of forked, freed and moved pages: worked examples, and what follows from the definitions."""
import random

from oracle import pages as OP


def test_a_fork_shares_full_pages_and_copies_the_last():
    kv_len, pages, table = [35, 0, 0, 32], [3, 0, 0, 3], [[7, 2, 9, -1], [-1] * 4, [5, 5, 5, 5], [1, 3, 8, -1]]
    got = OP.fork([0, 3], [1, 2], [20, 21], kv_len, table, pages)
    assert got == ([9, -1], [20, -1], [2, 1, 0])
    assert kv_len == [35, 35, 32, 32] and pages == [3, 3, 2, 3]
    assert table == [[7, 2, 9, -1], [7, 2, 20, -1], [1, 3, 5, 5], [1, 3, 8, -1]]


def test_pairs_that_are_refused():
    kv_len, pages, table = [20, 20, -1, 33, 5], [2, 1, 1, 4, 1], [[0, 1, -1]] * 5
    for src, dst, new in ((0, 0, 9), (0, 5, 9), (-1, 1, 9), (1, 4, 9), (2, 4, 9), (3, 4, 9), (0, 4, -1), (0, 4, 1 << 27)):
        assert OP.fork([src], [dst], [new], kv_len, table, pages) == ([-2], [-2], [0, 0, 1])
    assert OP.fork([0], [4], None, kv_len, table, pages)[2] == [0, 0, 1]
    # one place twice: the first; a place that another pair continues: not at all
    table = [[b, b + 10, -1] for b in range(5)]
    assert OP.fork([0, 0, 4], [1, 1, 2], [9, 8, 7], [20, 0, 0, 0, 4], table, [2, 0, 0, 0, 1])[2] == [2, 2, 1]
    assert OP.fork([0, 1], [1, 2], [9, 8], [20, 20, 0, 0, 4], table, [2, 2, 0, 0, 1])[2] == [1, 1, 1]


def test_what_is_free():
    assert OP.free([[3, 0, 5], [3, 9, 1]], [2, 3], 6) == ([2, 4, 5, -1, -1, -1], [3, 3, 4])
    assert OP.free([[3, 0, 5]], [0], 2) == ([0, 1], [2, 0, 0])


def test_moves_close_the_pool():
    got = OP.compact([[7, 0, -1], [7, 5, 2]], [2, 3], 8, 4)
    assert got == ([[1, 0, -1], [1, 3, 2]], [7, 5, -1, -1], [1, 3, -1, -1], [4, 2, 4])
    rng = random.Random(3)
    for _ in range(50):
        n = rng.randint(1, 60)
        table = [[rng.randrange(n) for _ in range(6)] for _ in range(4)]
        pages = [rng.randint(0, 6) for _ in range(4)]
        pool = [list(range(n)), [100 + p for p in range(n)]]
        for cap in (0, 2, n):
            after, a, b, (used, moves, last) = OP.compact(table, pages, n, cap)
            moved = [list(x) for x in pool]
            OP.copies(moved, a, b)
            for layer, was in zip(moved, pool):            # every entry still finds its page's contents
                assert [[layer[p] for p in row[:k]] for row, k in zip(after, pages)] == [[was[p] for p in row[:k]] for row, k in zip(table, pages)]
            assert last == used if cap == n else last >= used
            assert not set(a[:moves]) & set(b[:moves]) and max(OP.listed(after, pages, n), default=-1) + 1 == last
