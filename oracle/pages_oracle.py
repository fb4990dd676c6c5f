"""Oracle of the pages of a pool: which of them sequences share, get and give back, page by page from the definitions.  Tables are lists
of rows, or arrays; all results are lists."""


def _free(rows, held, n_pages):
    used = {p for row in rows for p in row if 0 <= p < n_pages}
    return [p for p in range(n_pages) if p not in used and not (held is not None and held[p] != 0)]


def fork(table, lens, parents, held, page_size, n_pages):
    """(new table, new lens, src, dst, missing)"""
    wide, rows, new_lens = len(table[0]), [], []
    for p in parents:
        n = min(max(int(lens[p]), 0), wide * page_size) if 0 <= p < len(table) else 0
        new_lens.append(n)
        rows.append([int(x) for x in table[p][:-(-n // page_size)]] if n else [])
    whole = {p for row, n in zip(rows, new_lens) for p in row[:n // page_size]}
    free, kept = _free(rows, held, n_pages), set()
    src, dst, missing = [], [], 0
    for row, n in zip(rows, new_lens):
        pair = (-1, -1)
        if n % page_size and 0 <= row[-1] < n_pages:
            if row[-1] in whole or row[-1] in kept or (held is not None and held[row[-1]] != 0):
                if free:
                    pair = (row[-1], free.pop(0))
                else:
                    missing += 1
                row[-1] = pair[1]
            else:
                kept.add(row[-1])
        src.append(pair[0])
        dst.append(pair[1])
        row += [-1] * (wide - len(row))
    return rows, new_lens, src, dst, missing


def extend(table, lens, counts, held, page_size, n_pages):
    """(table, missing)"""
    rows = [[int(x) for x in row] for row in table]
    free, missing = _free(rows, held, n_pages), 0
    for row, n, count in zip(rows, lens, counts):
        n = max(int(n), 0)
        for e in range(n // page_size, (n + int(count) - 1) // page_size + 1 if count > 0 else 0):
            if e >= len(row):
                missing += 1
            elif not 0 <= row[e] < n_pages:
                row[e] = free.pop(0) if free else -1
                missing += row[e] < 0
    return rows, missing


def compact(table, held, n_pages, moves):
    """(table, src, dst, top)"""
    rows = [[int(x) for x in row] for row in table]
    fixed = {p for p in range(n_pages) if held is not None and held[p] != 0}
    used = {p for row in rows for p in row if 0 <= p < n_pages}
    free, high, to = _free(rows, held, n_pages), sorted(used - fixed), {}
    while free and high and free[0] < high[-1] and len(to) < moves:
        to[high.pop()] = free.pop(0)
    rows = [[to.get(p, p) for p in row] for row in rows]
    src, dst = list(to.keys()), list(to.values())
    pad = [-1] * (moves - len(to))
    top = 1 + max(fixed | {to.get(p, p) for p in used}, default=-1)
    return rows, src + pad, dst + pad, top
