"""Oracle: the management of a paged cache's pages, one sequence and one page after the other (test
infrastructure).

A state is (rows, lens, refs): the pages of each sequence, as many as its tokens need, their
lengths, and a count per page. Functions return the new state, the moves, and the status bits
(1: a page number out of range, 2: a length or a parent out of range, 4: no page was free).
"""
from __future__ import annotations


def rows_of(table, lens, page: int):
    """A state's rows from a page table, with lengths outside of their row's cut off."""
    width = len(table[0]) if len(table) else 0
    cut = [min(max(n, 0), width * page) for n in lens]
    return [list(t[:-(-n // page)]) for t, n in zip(table, cut)], cut, 2 * (cut != list(lens))


def table_of(rows, width: int):
    return [list(r) + [-1] * (width - len(r)) for r in rows]


def _bad_pages(rows, n):
    return int(any(not 0 <= p < n for r in rows for p in r))


def fork(rows, lens, refs, parent):
    refs, n = list(refs), len(refs)
    status = _bad_pages(rows, n)

    def count(row, by):
        for p in row:
            if 0 <= p < n:
                refs[p] += by

    new, new_lens = [], []
    for b, p in enumerate(parent):
        if p >= len(rows):
            status |= 2
            p = -1
        new.append(list(rows[p]) if p >= 0 else [])
        new_lens.append(lens[p] if p >= 0 else 0)
        if p != b:
            count(rows[b], -1)
            count(new[b], 1)
    return new, new_lens, refs, status


def extend(rows, lens, refs, grow, page: int, width: int):
    free = [p for p, r in enumerate(refs) if r == 0]
    after, moves, taken, status, out = list(refs), [], 0, _bad_pages(rows, len(refs)), []
    lens = list(lens)
    for b, row in enumerate(rows):
        row = list(row)
        n = lens[b] + grow[b]
        if n < 0:
            status |= 2
            n = 0
        pages = -(-n // page)
        split = grow[b] > 0 and lens[b] % page > 0 and 0 <= row[-1] < len(refs) and refs[row[-1]] > 1
        need = max(0, pages - len(row)) + split
        first, taken = taken, taken + need
        fits = n <= width * page
        if not fits:
            status |= 2
        elif need and taken > len(free):
            status |= 4
            fits = False
        if fits:
            lens[b] = n
            mine = free[first:taken]
            if split:
                moves.append((row[-1], mine[0]))
                after[row[-1]] -= 1
                row[-1] = mine[0]
            for p in mine:
                after[p] += 1
            for p in row[pages:]:
                if 0 <= p < len(refs):
                    after[p] -= 1
            row = row[:pages] + mine[split:]
        out.append(row)
    return out, lens, after, moves, status


def compact(rows, refs):
    used = [p for p, r in enumerate(refs) if r != 0]
    u = len(used)
    into = [p for p in range(u) if refs[p] == 0]
    moves = list(zip([p for p in used if p >= u], into))
    to = {p: p for p in used}
    to.update(moves)
    counts = [0] * len(refs)
    for p in used:
        counts[to[p]] = refs[p]
    status = int(any(p not in to for r in rows for p in r))
    return [[to.get(p, -1) for p in r] for r in rows], counts, [to.get(p, -1) for p in range(len(refs))], moves, status
