"""Block tables and slots of a paged cache from the requests' lengths, one sequence after the other."""


def page_tables(kv_len, new_rows, held, free_pages, table, slots_cap, page=16):
    """table: list of lists, grown in place.  Returns (pages, row_off, slots, summary)."""
    cols, asked, reach, refused = len(table[0]), 0, 0, 0
    pages, row_off, slots = [], [0], []
    for b, (n, new, has) in enumerate(zip(kv_len, new_rows, held)):
        need = -(-max(n, 0) // page)
        fits = 0 <= new <= n and need <= cols and 0 <= has <= cols
        ask = max(0, need - has) if fits else 0
        first, asked = asked, asked + ask
        granted = fits and (ask == 0 or asked <= len(free_pages))
        if granted:
            table[b][has:has + ask] = free_pages[first:first + ask]
            reach = asked
        refused += not granted
        pages.append(max(need, has) if granted else has)
        for i in range(max(new, 0)):
            pos = n - new + i
            at = table[b][pos // page] if granted else -1
            slots.append(at * page + pos % page if 0 <= at < 1 << 27 else -1)
        row_off.append(len(slots))
    rows = len(slots)
    return pages, row_off, (slots + [-1] * slots_cap)[:slots_cap], [rows, reach, refused]
