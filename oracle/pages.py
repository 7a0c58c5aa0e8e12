"""Pages of a paged cache for new tokens and back, sequence by sequence, with Python's whole numbers."""


def pages_of(tokens, page):
    return -(-tokens // page)


def reserve(table, lens, new, free, counts, page, rows_cap):
    """table: lists of pages (changed in place); free: list, read only; counts: [free pages, ...].  Returns a dict like RolloutStage.reserve's."""
    width = len(table[0]) if table else 0
    most, n_pages = width * page, len(free)
    n_free = left = min(max(counts[0], 0), n_pages)
    asked, refused = 0, 0
    cu, start, out_lens, slots, positions = [0], [], [], [], []
    for i, (n, x) in enumerate(zip(lens, new)):
        n, x = min(max(n, 0), most), max(x, 0)
        end = cu[-1] + x
        fits = n + x <= most and (x == 0 or end <= rows_cap)
        need = pages_of(n + x, page) - pages_of(n, page) if fits else 0
        asked += need
        served = fits and (need == 0 or asked <= n_free)
        if served:
            for place in range(pages_of(n, page), pages_of(n + x, page)):
                left -= 1
                table[i][place] = free[left]
        refused += not served
        for j in range(min(x, max(0, rows_cap - cu[-1]))):
            t = n + j
            p = table[i][t // page] if served else -1
            slots.append(p * page + t % page if 0 <= p < n_pages else -1)
            positions.append(t)
        cu.append(end)
        start.append(n if served else -1)
        out_lens.append(n + x if served else n)
    pad = rows_cap - len(slots)
    return dict(slots=slots + [-1] * pad, position_ids=positions + [0] * pad, cu_new=[min(c, 2 ** 31 - 1) for c in cu], start=start, seq_lens=out_lens,
                counts=[left, refused])


def release(table, lens, keep, free, counts, page):
    """free is changed in place.  Returns (lengths, counts)."""
    width = len(table[0]) if table else 0
    n_pages = len(free)
    left, out = min(max(counts[0], 0), n_pages), []
    for i, (n, k) in enumerate(zip(lens, keep)):
        n = min(max(n, 0), width * page)
        k = min(max(k, 0), n)
        for place in range(pages_of(k, page), pages_of(n, page)):
            if 0 <= table[i][place] < n_pages and left < n_pages:
                free[left] = table[i][place]
                left += 1
        out.append(k)
    return out, [left, 0]
