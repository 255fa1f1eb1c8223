"""sss_page_fork by its definition, page by page: a partly filled last page has one holder in
the new table."""
import numpy as np


def fork(parents, past, page, free, table):
    """(new_table, new_past, src, dst, used).  Entries that are held are pages (>= 0)."""
    width = table.shape[1]
    lens = [past[p] if p >= 0 else 0 for p in parents]
    rows = [[int(x) for x in table[p][:-(-n // page)]] if p >= 0 else [] for p, n in zip(parents, lens)]
    whole = {x for row, n in zip(rows, lens) for x in row[:n // page]}  # pages that some row holds full
    kept, used, src, dst = set(), 0, [-1] * len(rows), [-1] * len(rows)
    for r, (row, n) in enumerate(zip(rows, lens)):
        if n % page == 0:
            continue
        if row[-1] in whole or row[-1] in kept:
            src[r], dst[r] = row[-1], int(free[used])
            row[-1] = dst[r]
            used += 1
        else:
            kept.add(row[-1])
    rows = [row + [-1] * (width - len(row)) for row in rows]
    return [np.array(x, np.int64) for x in (rows, lens, src, dst, [used])]
