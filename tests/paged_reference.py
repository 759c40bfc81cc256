"""Planning pages, by its definition, with lists."""


def plan(tables, lens, free, page_rows, want):
    """tables: lists of pages per segment (as many as max_pages), lens, free: the stack, want: lengths.  Returns tables, lens, free,
    the rows that come in [(segment, row)], whether everything fitted."""
    tables, free = [list(t) for t in tables], list(free)
    most = len(tables[0]) * page_rows
    have = [-(-min(max(n, 0), most) // page_rows) for n in lens]
    cut = [min(max(w, 0), most) for w in want]
    need = [-(-w // page_rows) for w in cut]
    gone = [tables[s][i] for s in range(len(lens)) for i in range(need[s], have[s])]
    free += gone[::-1]
    new, rows, fits = [], [], True
    for s in range(len(lens)):
        got = min(have[s], need[s])
        for i in range(have[s], need[s]):
            if not free:
                break
            tables[s][i] = free.pop()
            got += 1
        n = min(cut[s], got * page_rows)
        fits &= n == cut[s]
        new.append(n)
        rows += [(s, r) for r in range(min(max(lens[s], 0), most), n)]
    return tables, new, free, rows, fits
