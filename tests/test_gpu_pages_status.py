"""The status bits of the page calls: every entry that a sequence holds and every length, of sequences that stay, end,
are taken over, grow and shrink alike."""
import numpy as np
import pytest

from oracle import pages as op
from test_gpu_pages import _moves, _Pool

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

N, PAGE, BATCH, WIDTH = 20, 16, 4, 3
TABLE = [[0, 1, 2], [3, 4, 5], [6, 7, 8], [9, 10, 11]]
LENS = [40, 33, 16, 0]  # entries held: 3, 3, 1, 0
REFS = [1] * 7 + [0] * 13
# (sequence, entry, page) that are put into the table, lengths that replace others, the bits of both
TABLES = {
    "as they should be": ([], {}, 0),
    "behind the ends": ([(2, 1, 99), (2, 2, -5), (3, 0, 20)], {}, 0),
    "the first entry": ([(0, 0, -1)], {}, 1),
    "one in the middle": ([(1, 1, N)], {}, 1),
    "the last, partly filled": ([(1, 2, 1 << 30)], {}, 1),
    "the only one": ([(2, 0, -(1 << 31))], {}, 1),
    "too long": ([], {1: WIDTH * PAGE + 1}, 2),
    "too long, and not its pages": ([(1, 0, 20)], {1: 1 << 30}, 3),
    "below zero": ([], {2: -1}, 2),
}
PARENTS = {"all stay": [0, 1, 2, 3], "all end": [-1, -1, -1, -1], "one ends": [0, -1, 2, 3], "another ends": [0, 1, -1, 3],
           "taken over": [1, 1, 2, 2], "exchanged": [1, 2, 0, 3]}
GROWTH = {"nothing": [0, 0, 0, 0], "a token": [1, 1, 1, 1], "fewer": [-3, -17, -1, 0], "all of it": [-40, -33, -16, 0],
          "no room": [8, 15, 32, 48]}


def _state(name):
    changes, lens, bits = TABLES[name]
    table = [list(r) for r in TABLE]
    for b, s, p in changes:
        table[b][s] = p
    lens = [lens.get(b, x) for b, x in enumerate(LENS)]
    rows, cut, _ = op.rows_of(table, lens, PAGE)
    return table, lens, rows, cut, bits


@pytest.mark.parametrize("parent", PARENTS)
@pytest.mark.parametrize("name", TABLES)
def test_fork(name, parent):
    table, lens, rows, cut, bits = _state(name)
    new, l1, r1, pages = op.fork(rows, cut, REFS, PARENTS[parent])
    assert pages == bits & 1  # (of every sequence, whatever becomes of it)
    got = _Pool(N, PAGE, BATCH, WIDTH).fork(table, lens, REFS, PARENTS[parent])
    assert got == [op.table_of(new, WIDTH), l1, r1, bits]


@pytest.mark.parametrize("free", [13, 1, 0])
@pytest.mark.parametrize("grow", GROWTH)
@pytest.mark.parametrize("name", TABLES)
def test_extend(name, grow, free):
    table, lens, rows, cut, bits = _state(name)
    refs = REFS[:7] + [1] * (13 - free) + [0] * free
    new, l1, r1, moves, more = op.extend(rows, cut, refs, GROWTH[grow], PAGE, WIDTH)
    assert more & 1 == bits & 1
    got = _Pool(N, PAGE, BATCH, WIDTH).extend(table, lens, refs, GROWTH[grow])
    assert got == [op.table_of(new, WIDTH), l1, r1, _moves(moves, BATCH), [len(moves)], bits | more]


@pytest.mark.parametrize("name", TABLES)
def test_compact(name):
    table, lens, rows, cut, bits = _state(name)
    refs = REFS[:9] + [1] + REFS[10:]  # (page 9 moves)
    new, r1, renamed, moves, pages = op.compact(rows, refs)
    assert pages == bits & 1
    got = _Pool(N, PAGE, BATCH, WIDTH).compact(table, lens, refs)
    assert got == [op.table_of(new, WIDTH), r1, renamed, _moves(moves, N // 2), [len(moves)], bits | pages]


@pytest.mark.parametrize("at", [0, 1023, 1024, 2000, 2499])
def test_an_entry_far_in_a_row(at):
    n, width = 3000, 2500
    table = np.arange(width)[None].repeat(2, axis=0)
    table[1, at] = n
    lens, refs = [0, width * 16], [1] * width + [0] * 500
    refs[at] = 0
    pool = _Pool(n, 16, 2, width)
    rows = op.rows_of(table.tolist(), lens, 16)[0]
    new, l1, r1, bits = op.fork(rows, lens, refs, [0, 1])
    assert pool.fork(table, lens, refs, [0, 1]) == [op.table_of(new, width), l1, r1, bits] and bits == 1
    new, l1, r1, moves, bits = op.extend(rows, lens, refs, [0, 0], 16, width)
    assert pool.extend(table, lens, refs, [0, 0]) == [op.table_of(new, width), l1, r1, _moves(moves, 2), [0], bits] and bits == 1
