"""The management of a cache's pages on the host: the oracle's own pins, refusals (nothing is queued),
and the kernels' assembly."""
import os

import pytest

import paper_2601_20595_amd as csg
from oracle import pages as op
from test_kernel_asm import device_asm, divergent_barrier_loops, wide_stores_with_offset_register

P = 1 << 20
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED = csg.CSG_ERR_INVALID, csg.CSG_ERR_UNSUPPORTED


def _cfg(**change):
    c = csg.csg_pages_cfg(n_pages=10, page_size=16, batch=2, max_pages=4)
    for k, v in change.items():
        setattr(c, k, v)
    return c


def _status(f, *args, **kw):
    with pytest.raises(csg.CsgError) as e:
        f(*args, **kw)
    return e.value.status


def _at(n, first=P):
    """Addresses far enough apart that no two buffers overlap."""
    return [first + (i << 16) for i in range(n)]


def test_oracle_by_hand():
    # two sequences of 20 and 16 tokens in pages of 16: pages 3, 1 and 2
    rows, lens, bits = op.rows_of([[3, 1, 9], [2, 9, 9]], [20, 16], 16)
    refs = [0, 1, 1, 1, 0, 0]
    assert (rows, lens, bits) == ([[3, 1], [2]], [20, 16], 0)
    # both become the first one
    rows, lens, refs, bits = op.fork(rows, lens, refs, [0, 0])
    assert (rows, lens, refs, bits) == ([[3, 1], [3, 1]], [20, 20], [0, 2, 0, 2, 0, 0], 0)
    # each copies the shared last page; 0 and 2 are the lowest free ones, then 4 for a new page
    rows, lens, refs, moves, bits = op.extend(rows, lens, refs, [1, 13], 16, 3)
    assert (rows, lens, refs) == ([[3, 0], [3, 2, 4]], [21, 33], [1, 0, 1, 2, 1, 0])
    assert (moves, bits) == ([(1, 0), (1, 2)], 0)
    # four pages are in use: 4 goes to 1
    rows, refs, renamed, moves, bits = op.compact(rows, refs)
    assert (rows, refs, renamed, moves, bits) == ([[3, 0], [3, 2, 1]], [1, 1, 1, 2, 0, 0], [0, -1, 2, 3, 1, -1], [(4, 1)], 0)
    # one page too few for the second; the third, which asks for none, grows
    got = op.extend([[0], [1], [2]], [16, 16, 3], [1, 1, 1, 0], [1, 1, 2], 16, 4)
    assert got == ([[0, 3], [1], [2]], [17, 16, 5], [1, 1, 1, 1], [], 4)
    # too long for its row; more given back than there is
    assert op.extend([[0], [1]], [16, 3], [1, 1, 0], [1, -4], 16, 1) == ([[0], []], [16, 0], [1, 0, 0], [], 2)


BAD = [({"n_pages": 0}, INVALID), ({"n_pages": (1 << 24) + 1}, UNSUPPORTED), ({"page_size": 0}, INVALID), ({"page_size": 24}, UNSUPPORTED),
       ({"batch": -1}, INVALID), ({"batch": (1 << 20) + 1}, UNSUPPORTED), ({"max_pages": 0}, INVALID),
       ({"max_pages": (1 << 26) + 1}, UNSUPPORTED), ({"max_pages": 1 << 25, "batch": 1 << 15}, UNSUPPORTED), ({"reserved": 1}, INVALID)]


@pytest.mark.parametrize("change, status", BAD)
def test_refuses(change, status):
    c = _cfg(**change)
    assert _status(csg.csg_pages_workspace, c) == status
    assert _status(csg.csg_pages_fork, c, *_at(7)) == status
    assert _status(csg.csg_pages_extend, c, *_at(10), 1 << 40) == status
    assert _status(csg.csg_pages_compact, c, *_at(9), 1 << 40) == status


def test_refuses_buffers():
    c = _cfg()
    need = csg.csg_pages_workspace(c)
    for f, n, tail in ((csg.csg_pages_fork, 7, ()), (csg.csg_pages_extend, 10, (need,)), (csg.csg_pages_compact, 9, (need,))):
        for i in range(n):
            args = _at(n)
            args[i] = 0
            assert _status(f, c, *args, *tail) == INVALID
    # a short or crooked workspace
    for f, n in ((csg.csg_pages_extend, 10), (csg.csg_pages_compact, 9)):
        assert _status(f, c, *_at(n), need - 1) == INVALID
        args = _at(n)
        args[-1] += 4
        assert _status(f, c, *args, need) == INVALID
    # outputs that meet inputs, or each other (their last word and the next one's first)
    for f, n, ins, outs, tail in ((csg.csg_pages_fork, 7, 4, range(4, 7), ()), (csg.csg_pages_extend, 10, 4, range(4, 10), (need,)),
                                  (csg.csg_pages_compact, 9, 3, range(3, 9), (need,))):
        for o in outs:
            for i in list(range(ins)) + [x for x in outs if x != o]:
                args = _at(n)
                args[o] = args[i]
                assert _status(f, c, *args, *tail) == INVALID, (f, o, i)
    args = _at(7)
    args[4] = args[0] + 4 * (2 * 4 - 1)
    assert _status(csg.csg_pages_fork, c, *args) == INVALID
    for f, n, tail in ((csg.csg_pages_fork, 7, ()), (csg.csg_pages_extend, 10, (need,)), (csg.csg_pages_compact, 9, (need,))):
        assert _status(f, c, *_at(n), *tail, device=64) == INVALID


def test_copy_refuses():
    a, b = _at(2)
    assert _status(csg.csg_pages_copy, 0, 64, [a], b, 3, b) == INVALID
    assert _status(csg.csg_pages_copy, 4, 24, [a], b, 3, b) == INVALID
    assert _status(csg.csg_pages_copy, 4, -16, [a], b, 3, b) == INVALID
    assert _status(csg.csg_pages_copy, 4, (1 << 31) + 16, [a], b, 3, b) == UNSUPPORTED
    assert _status(csg.csg_pages_copy, 4, 64, [a], b, -1, b) == INVALID
    assert _status(csg.csg_pages_copy, 4, 64, [a, 0], b, 3, b) == INVALID
    assert _status(csg.csg_pages_copy, 4, 64, [a, a + 8], b, 3, b) == INVALID
    assert _status(csg.csg_pages_copy, 4, 64, [a], 0, 3, b) == INVALID
    assert _status(csg.csg_pages_copy, 4, 64, [a], b, 3, 0) == INVALID
    assert _status(csg.csg_pages_copy, 4, 64, [a], b, 3, b, device=64) == INVALID
    # nothing to do
    csg.csg_pages_copy(4, 64, [], b, 3, b)
    csg.csg_pages_copy(4, 64, [a], 0, 0, 0)
    csg.csg_pages_copy(4, 0, [a], b, 3, b)


def test_python_refuses():
    torch = pytest.importorskip("torch")
    pool = csg.PagePool(10, 16, 2, 4)
    t, n, r = (torch.zeros(s, dtype=torch.int32) for s in ((2, 4), (2,), (10,)))
    with pytest.raises(ValueError, match="GPU"):
        pool.fork(t, n, r, n, t, n, r)
    with pytest.raises(ValueError, match="4 pages"):
        pool.fork(t[:, :3], n, r, n, t, n, r)
    with pytest.raises(ValueError, match="int32"):
        pool.fork(t.float(), n, r, n, t, n, r)
    with pytest.raises(ValueError, match="same size"):
        pool.copy([torch.zeros(10, 16), torch.zeros(10, 32)], t, n)
    with pytest.raises(ValueError, match="10, ..."):
        pool.copy([torch.zeros(9, 16)], t, n)
    with pytest.raises(csg.CsgError):
        csg.PagePool(10, 24, 2, 4)


def test_kernels_assembly():
    asm = device_asm(os.path.join(ROOT, "paper_2601_20595_amd", "csrc", "pages.hip"))
    assert divergent_barrier_loops(asm) == []
    assert wide_stores_with_offset_register(asm) == []
    assert "scratch_" not in asm, "a kernel spills"
