"""Pages of a paged cache that are forked, counted and moved, one sequence after the other."""


def fork(src, dst, new_pages, kv_len, table, pages, page=16):
    """kv_len, table (list of lists) and pages are changed in place.  Returns (copy_from, copy_to, summary)."""
    batch, cols = len(kv_len), len(table[0])
    copy_from, copy_to, done = [-2] * len(src), [-2] * len(src), []
    for i, (s, d) in enumerate(zip(src, dst)):
        if not (0 <= s < batch and 0 <= d < batch) or s == d or d in dst[:i] or d in src:
            continue
        need = -(-kv_len[s] // page) if kv_len[s] >= 0 else cols + 1
        part = kv_len[s] % page != 0
        if need > pages[s] or pages[s] > cols or (part and not (new_pages is not None and 0 <= new_pages[i] < 1 << 27)):
            continue
        done.append((i, s, d, need, part))
    for i, s, d, need, part in done:
        kv_len[d], pages[d] = kv_len[s], need
        copy_from[i] = copy_to[i] = -1
        table[d][:need] = table[s][:need]
        if part:
            copy_from[i], copy_to[i] = table[s][need - 1], new_pages[i]
            table[d][need - 1] = new_pages[i]
    return copy_from, copy_to, [len(done), sum(x[4] for x in done), len(src) - len(done)]


def copies(pool, copy_from, copy_to):
    """pool: [layers][pages] of anything, changed in place."""
    n = len(pool[0])
    for a, b in zip(copy_from, copy_to):
        if 0 <= a < n and 0 <= b < n and a != b:
            for layer in pool:
                layer[b] = layer[a]


def listed(table, pages, n_pages):
    """The pages of the pool that the tables' entries list, an entry each."""
    return [p for row, n in zip(table, pages) for p in row[:max(n, 0)] if 0 <= p < n_pages]


def free(table, pages, n_pages):
    """(free pages ascending, then -1; summary)"""
    entries = listed(table, pages, n_pages)
    left = sorted(set(range(n_pages)) - set(entries))
    return left + [-1] * (n_pages - len(left)), [len(left), n_pages - len(left), len(entries)]


def compact(table, pages, n_pages, max_moves):
    """(table afterwards, copy_from, copy_to, summary)"""
    used = set(listed(table, pages, n_pages))
    far = sorted((p for p in used if p >= len(used)), reverse=True)[:max_moves]
    holes = [p for p in range(len(used)) if p not in used][:max_moves]
    now = dict(zip(far, holes))
    after = [[now.get(p, p) for p in row[:max(n, 0)]] + row[max(n, 0):] for row, n in zip(table, pages)]
    pad = [-1] * (max_moves - len(far))
    last = max((now.get(p, p) for p in used), default=-1) + 1
    return after, far + pad, holes[:len(far)] + pad, [len(used), len(far), last]
