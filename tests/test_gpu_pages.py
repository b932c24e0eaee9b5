"""The management of a cache's pages on the GPU against the oracle, every number equal, and a run of
it with the caches that it serves."""
import os
import re

import numpy as np
import pytest

import paper_2601_20595_amd as csg
from oracle import cache4
from oracle import doc_attention as oda
from oracle import pages as op

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from attn_util import DEV, HALF_STEP, TINY, TORCH, close, f64, ints, normal, pointers
    from cache4_util import pages4

pytestmark = pytest.mark.gpu


def _state(rng, n_pages, page, batch, width, fill):
    """(table, lens, refs): prefixes shared by neighbours, some pages held by the caller too."""
    order = list(rng.permutation(n_pages)[:int(n_pages * fill)])
    rows, lens = [], []
    for b in range(batch):
        n = int(rng.integers(0, min(width * page, 2 * (len(order) // max(1, batch - b)) * page + page) + 1))
        need = -(-n // page)
        row = []
        if rows and rng.random() < 0.4:
            row = list(rows[-1][:int(rng.integers(0, len(rows[-1]) + 1))])[:need]
        while len(row) < need and order:
            row.append(int(order.pop()))
        n = min(n, len(row) * page)
        rows.append(row[:-(-n // page)])
        lens.append(n)
    refs = np.zeros(n_pages, dtype=int)
    for r in rows:
        for p in r:
            refs[p] += 1
    for p in order[:len(order) // 2]:
        refs[p] += int(rng.integers(1, 3))
    table = np.full((batch, width), 12345678, dtype=np.int32)  # (behind a sequence's end: anything)
    for b, r in enumerate(rows):
        table[b, :len(r)] = r
    return table, lens, refs


class _Pool:
    """The calls on host arrays; outputs begin as 77."""

    def __init__(self, n_pages, page, batch, width):
        self.pool = csg.PagePool(n_pages, page, batch, width)
        self.n, self.page, self.batch, self.width = n_pages, page, batch, width
        self.ws = torch.full((self.pool.workspace_bytes(),), 255, dtype=torch.uint8, device=DEV)

    def _new(self, *shape):
        return torch.full(shape, 77, dtype=torch.int32, device=DEV)

    def _run(self, f, ins, outs, *more):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        dev = [torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV) for x in ins]
        dev[0] = dev[0].reshape(self.batch, self.width)
        f(*dev, *outs, *more, status=st)
        torch.cuda.synchronize()
        return [x.cpu().numpy().tolist() for x in outs] + [int(st)]

    def fork(self, table, lens, refs, parent):
        return self._run(self.pool.fork, (table, lens, refs, parent), (self._new(self.batch, self.width), self._new(self.batch), self._new(self.n)))

    def extend(self, table, lens, refs, grow):
        return self._run(self.pool.extend, (table, lens, refs, grow),
                         (self._new(self.batch, self.width), self._new(self.batch), self._new(self.n), self._new(self.batch, 2), self._new(1)), self.ws)

    def compact(self, table, lens, refs):
        return self._run(self.pool.compact, (table, lens, refs),
                         (self._new(self.batch, self.width), self._new(self.n), self._new(self.n), self._new(self.n // 2, 2), self._new(1)), self.ws)


def _moves(moves, room):
    return [list(m) for m in moves] + [[77, 77]] * (room - len(moves))


# pages, page size, sequences, entries of a row, share of the pages that may be in use
SIZES = [(1, 16, 1, 1, 1.0), (7, 16, 3, 4, 0.8), (40, 32, 12, 9, 0.7), (300, 64, 30, 20, 0.9), (4095, 16, 70, 90, 0.8), (4096, 16, 5, 1030, 0.6),
         (4097, 128, 300, 40, 0.95), (20000, 16, 257, 1024, 0.5), (70001, 256, 1000, 60, 0.4), (64, 16, 0, 5, 0.5)]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("seed", [0, 1])
def test_against_the_oracle(size, seed):
    n, page, batch, width, fill = size
    rng = np.random.default_rng(seed + 10 * n)
    table, lens, refs = _state(rng, n, page, batch, width, fill)
    pool = _Pool(n, page, batch, width)
    rows = op.rows_of(table.tolist(), lens, page)[0]
    # fork: some stay, some end, some take a neighbour's place
    parent = [int(rng.choice([b, b, -1 - (b % 3), rng.integers(0, batch)])) for b in range(batch)]
    got = pool.fork(table, lens, refs, parent)
    new, lens1, refs1, bits = op.fork(rows, lens, refs.tolist(), parent)
    assert got == [op.table_of(new, width), lens1, refs1, bits] and bits == 0
    # extend: by a token, by many, back, by nothing
    grow = [int(rng.choice([0, 1, 1, 1, rng.integers(1, 4 * page), -rng.integers(0, x + 1)])) for x in lens1]
    got = pool.extend(got[0], got[1], got[2], grow)
    new, lens2, refs2, moves, bits = op.extend(new, lens1, refs1, grow, page, width)
    assert got == [op.table_of(new, width), lens2, refs2, _moves(moves, batch), [len(moves)], bits]
    # compact
    got = pool.compact(got[0], got[1], got[2])
    new, refs3, renamed, moves, bits = op.compact(new, refs2)
    assert got == [op.table_of(new, width), refs3, renamed, _moves(moves, n // 2), [len(moves)], bits] and bits == 0


def test_no_page_is_free_and_rows_that_are_full():
    pool = _Pool(4, 16, 4, 2)
    table, lens, refs = [[0, 9], [1, 9], [2, 9], [3, 9]], [16, 16, 3, 16], [1, 1, 1, 1]
    state = op.rows_of(table, lens, 16)[0]
    for refs in ([1, 1, 1, 1], [2, 1, 2, 0]):
        for grow in ([1, 1, 5, 1], [0, 17, 1, 0], [-17, 0, 0, 40], [2147483647] * 4, [-2147483648] * 4, [0, -16, 0, 1]):
            new, l2, r2, moves, bits = op.extend(state, lens, refs, grow, 16, 2)
            assert pool.extend(table, lens, refs, grow) == [op.table_of(new, 2), l2, r2, _moves(moves, 4), [len(moves)], bits], (refs, grow)


def test_bad_tables_set_bits_and_touch_nothing_else():
    n, page, batch, width = 50, 16, 4, 6
    pool = _Pool(n, page, batch, width)
    table = [[3, 50, -1, 7, 1, 2], [4, 5, 1 << 30, 8, 9, 6], [10, 11, 12, 13, 14, 15], [-5, -6, 0, 0, 0, 0]]
    lens = [40, 33, 5000, -3]
    refs = [1] * 25 + [0] * 25
    got = pool.fork(table, lens, refs, [1, 0, 4, 2])
    rows, cut, _ = op.rows_of(table, lens, page)
    new, l1, r1, bits = op.fork(rows, cut, refs, [1, 0, 4, 2])
    assert got == [op.table_of(new, width), l1, r1, 3]
    assert bits == 3
    got = pool.extend(table, lens, refs, [8, -30, 0, 1])
    new, l1, r1, moves, _ = op.extend(rows, cut, refs, [8, -30, 0, 1], page, width)
    assert got == [op.table_of(new, width), l1, r1, _moves(moves, batch), [len(moves)], 3]
    got = pool.compact(table, lens, refs)
    new, r1, renamed, moves, _ = op.compact(rows, refs)
    assert got == [op.table_of(new, width), r1, renamed, _moves(moves, n // 2), [len(moves)], 3]


def test_counts_that_do_not_hold_touch_no_memory_outside():
    """Rows that hold pages which the counts call free, twice the same page: the results' sizes and guards stay."""
    n, page, batch, width = 5000, 16, 40, 300
    rng = np.random.default_rng(0)
    pool = csg.PagePool(n, page, batch, width)
    table = ints(rng.integers(-3, n + 3, (batch, width)).tolist())
    lens = ints(rng.integers(-10, width * page + 10, batch).tolist())
    refs = ints(rng.integers(-1, 2, n).tolist())
    words = {"table": batch * width, "lens": batch, "refs": n, "renamed": n, "moves": 2 * batch, "cmoves": n // 2 * 2, "n_moves": 1}
    mem = {k: torch.full((v + 128,), 77, dtype=torch.int32, device=DEV) for k, v in words.items()}
    out = {k: mem[k][64:64 + v] for k, v in words.items()}
    ws = torch.zeros(pool.workspace_bytes() + 512, dtype=torch.uint8, device=DEV)
    w = ws[256:-256]
    change = ints(rng.integers(-5, 45, batch).tolist())
    t = out["table"].view(batch, width)
    pool.fork(table, lens, refs, change, t, out["lens"], out["refs"])
    pool.extend(table, lens, refs, change, t, out["lens"], out["refs"], out["moves"], out["n_moves"], w)
    pool.compact(table, lens, refs, t, out["refs"], out["renamed"], out["cmoves"], out["n_moves"], w)
    torch.cuda.synchronize()
    for k, m in mem.items():
        assert bool((m[:64] == 77).all()) and bool((m[64 + words[k]:] == 77).all()), k
    assert bool((ws[:256] == 0).all()) and bool((ws[-256:] == 0).all())


@pytest.mark.parametrize("page_bytes,buffers", [(16, 1), (544, 3), (16384, 2), (17408 * 3, 4), (131072, 2), (1040, 70)])
def test_copy(page_bytes, buffers):
    n = 40
    g = torch.Generator(device=DEV).manual_seed(1)
    data = [torch.randint(0, 256, (n, page_bytes), generator=g, device=DEV).to(torch.uint8) for _ in range(buffers)]
    order = np.random.default_rng(2).permutation(n)
    pool = csg.PagePool(n, 16, 1, 1)
    for count, room in ((7, 20), (0, 20), (20, 20), (-3, 20), (25, 20)):
        pairs = np.stack([order[:20], order[20:]], axis=1)
        want = [d.clone() for d in data]
        m = min(max(count, 0), room)
        for w in want:
            w[torch.tensor(pairs[:m, 1], device=DEV)] = w[torch.tensor(pairs[:m, 0], device=DEV)]
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        pool.copy(data, ints(pairs.tolist()), ints([count]), status=st)
        torch.cuda.synchronize()
        assert int(st) == 0 and all(torch.equal(a, b) for a, b in zip(data, want)), count
    bad = [[3, 40], [-1, 4], [5, 6], [1 << 30, 7]]
    want = [d.clone() for d in data]
    for w in want:
        w[6] = w[5]
    pool.copy(data, ints(bad), ints([4]), status=st)
    torch.cuda.synchronize()
    assert int(st) == 1 and all(torch.equal(a, b) for a, b in zip(data, want))


def test_far_pages_are_copied():
    """Pages beyond 2^32 bytes."""
    n, size = 34000, 131072
    data = torch.zeros((n, size), dtype=torch.uint8, device=DEV)
    data[n - 1] = 5
    data[1] = 9
    csg.PagePool(n, 16, 1, 1).copy([data], ints([[n - 1, 0], [1, n - 2]]), ints([2]))
    torch.cuda.synchronize()
    assert bool((data[0] == 5).all()) and bool((data[n - 2] == 9).all()) and bool((data[n - 3] == 0).all())


def test_captured_and_replayed():
    """A step as one graph (fork, extend, copy, compact, copy), replayed on other states."""
    n, page, batch, width = 400, 16, 24, 12
    pool = csg.PagePool(n, page, batch, width)
    rng = np.random.default_rng(4)
    ins = [ints(np.zeros(s, dtype=int).tolist()) for s in ((batch, width), batch, n, batch, batch)]
    new = lambda *s: torch.full(s, 77, dtype=torch.int32, device=DEV)
    mid, out, end = ([new(batch, width), new(batch), new(n)] for _ in range(3))
    moves, n_moves, moves2, n_moves2, renamed = new(batch, 2), new(1), new(n // 2, 2), new(1), new(n)
    ws = torch.zeros(pool.workspace_bytes(), dtype=torch.uint8, device=DEV)
    data = [torch.arange(n, dtype=torch.int32, device=DEV)[:, None].repeat(1, 1000) for _ in range(2)]
    results = [*mid, *out, end[0], end[2], renamed, n_moves, n_moves2, moves, moves2, *data]

    def step(stream):
        pool.fork(ins[0], ins[1], ins[2], ins[3], *mid, stream=stream)
        pool.extend(*mid, ins[4], *out, moves, n_moves, ws, stream=stream)
        pool.copy(data, moves, n_moves, stream=stream)
        pool.compact(*out, end[0], end[2], renamed, moves2, n_moves2, ws, stream=stream)
        pool.copy(data, moves2, n_moves2, stream=stream)

    st = torch.cuda.Stream(device=DEV)
    torch.cuda.synchronize()
    step(st)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        step(st)
    for _ in range(4):
        table, lens, refs = _state(rng, n, page, batch, width, 0.7)
        parent = [int(rng.choice([b, -1, rng.integers(0, batch)])) for b in range(batch)]
        for x, y in zip(ins, (table, lens, refs, parent, rng.integers(-3, 30, batch))):
            x.copy_(torch.tensor(np.asarray(y), dtype=torch.int32))
        got = []
        for graph in (True, False):
            for m in (moves, moves2):
                m.fill_(77)
            for d in data:
                d.copy_(torch.arange(n, dtype=torch.int32, device=DEV)[:, None].repeat(1, 1000))
            torch.cuda.synchronize()
            g.replay() if graph else step(None)
            torch.cuda.synchronize()
            got.append([x.clone() for x in results])
        assert all(torch.equal(a, b) for a, b in zip(*got))
        rows, cut, _ = op.rows_of(table.tolist(), lens, page)
        rows, cut, counts, _ = op.fork(rows, cut, refs.tolist(), parent)
        rows, cut, counts, m1, _ = op.extend(rows, cut, counts, ins[4].tolist(), page, width)
        held = list(range(n))
        for a, b in m1:
            held[b] = held[a]
        rows, counts, _, m2, _ = op.compact(rows, counts)
        for a, b in m2:
            held[b] = held[a]
        assert end[0].tolist() == op.table_of(rows, width) and end[2].tolist() == counts
        assert all(d[:, 0].tolist() == held and d[:, -1].tolist() == held for d in data)


@pytest.mark.parametrize("bits", [16, 4])
def test_a_serving_run(bits):
    """Prompts, sampled in forks, drafts taken back, ends, a compaction: every step's attention over the managed cache is
    that of plain lists of the sequences' tokens."""
    H, Hkv, D, page, batch, width, n, dtype = 4, 2, 64, 16, 6, 8, 40, "bf16"
    rng = np.random.default_rng(6)
    kind = csg.PagedCache if bits == 16 else csg.PagedCache4
    cache = kind(H, Hkv, D, dtype, n, page, batch, width)
    pool = csg.PagePool(n, page, batch, width)
    shape = (n, Hkv, page, D) if bits == 16 else (n, Hkv, page * (D // 2 + D // 32))
    kp, vp = (torch.zeros(shape, dtype=TORCH[dtype] if bits == 16 else torch.uint8, device=DEV) for _ in range(2))
    new = lambda *s: torch.full(s, -1, dtype=torch.int32, device=DEV)
    now, mid = ([new(batch, width), new(batch).zero_(), new(n).zero_()] for _ in range(2))
    moves, n_moves, renamed, st = new(n, 2), new(1), new(n), new(1).zero_()
    ws = torch.zeros(pool.workspace_bytes(), dtype=torch.uint8, device=DEV)
    text = [[] for _ in range(batch)]  # each token's key and value, as the cache holds them
    u = HALF_STEP[dtype]
    steps = [([0, 1, -1, -1, -1, -1], [37, 20, 0, 0, 0, 0]),  # two prompts
             ([0, 0, 0, 1, 1, -1], [1, 1, 1, 1, 1, 5]),        # forked; a third prompt
             ([0, 1, 2, 3, 4, 5], [4, 1, 4, 1, 0, 1]),         # drafts
             ([0, 1, 2, 3, 4, 5], [-3, 1, -2, 1, 1, 1]),       # taken back
             ([2, 2, -1, 3, 3, 5], [1, 1, 0, 12, 1, 13]),
             ([0, 1, 5, 5, -1, -1], [16, 17, 1, 1, 30, 0])]
    for t, (parent, grow) in enumerate(steps):
        pool.fork(*now, ints(parent), *mid, status=st)
        pool.extend(*mid, ints(grow), *now, moves, n_moves, ws, status=st)
        pool.copy([kp, vp], moves, n_moves, status=st)
        if t % 2:  # (out of place: table and counts into mid, lengths stay)
            pool.compact(*now, mid[0], mid[2], renamed, moves, n_moves, ws, status=st)
            pool.copy([kp, vp], moves, n_moves, status=st)
            now, mid = [mid[0], now[1], mid[2]], [now[0], mid[1], now[2]]
        text = [list(text[p]) if p >= 0 else [] for p in parent]
        fresh = [max(0, g) for g in grow]
        for b, g in enumerate(grow):
            if g < 0:
                del text[b][g:]
        m = sum(fresh)
        x, x64 = normal(30 + t, (m, H + 2 * Hkv, D), dtype)
        held = x64 if bits == 16 else cache4.values(*cache4.quantise(x64, dtype))
        at = pointers(fresh)
        for b in range(batch):
            text[b] += [(held[i, H:H + Hkv], held[i, H + Hkv:]) for i in range(at[b], at[b + 1])]
        xd = x.to(DEV)
        o, lse = torch.empty((m, H, D), dtype=TORCH[dtype], device=DEV), torch.empty((H, m), device=DEV)
        ws2 = torch.empty(cache.workspace_bytes(m), dtype=torch.uint8, device=DEV)
        ptr = ints(at)
        cache.append(kp, vp, xd[:, H:H + Hkv], xd[:, H + Hkv:], ptr, now[1], now[0], status=st)
        cache.attn(xd[:, :H], kp, vp, ptr, now[1], now[0], o, lse, ws2, status=st)
        torch.cuda.synchronize()
        assert int(st) == 0
        assert now[1].tolist() == [len(y) for y in text]
        counts = np.zeros(n, dtype=int)
        for b, row in enumerate(now[0].tolist()):
            assert [p >= 0 for p in row] == [i < -(-len(text[b]) // page) for i in range(width)]
            for p in row:
                if p >= 0:
                    counts[p] += 1
        assert now[2].tolist() == counts.tolist()
        for b in range(batch):
            if fresh[b]:
                k, v = (np.stack([y[i] for y in text[b]]) for i in range(2))
                r = slice(at[b], at[b + 1])
                want = oda.attention(x64[r, :H], k, v, oda.Scores(), 0, u, TINY[dtype])
                close(o[r], want[0], want[2], "o")
                close(lse[:, r], want[1], want[3], "lse")


def test_readme_example():
    """The serving example of README.md runs: both samples end with the prompt and two tokens, their first pages shared, and the
    last step's attention is that of what their caches hold."""
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    blocks = re.findall(r"```py3\n(.*?)```", text, re.S)
    assert len(blocks) == 1
    x = {}
    exec(compile(blocks[0], "README.md", "exec"), x)
    torch.cuda.synchronize()
    assert x["lens"].tolist() == [302, 302]
    rows = x["table"].tolist()
    assert rows[0][:4] == rows[1][:4] and rows[0][4] != rows[1][4] and rows[0][5:] == [-1] * 11
    k, v = (torch.empty((604, 8, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    x["cache"].read(x["k_pages"], x["v_pages"], ints([0, 302, 604]), x["lens"], x["table"], k, v)
    torch.cuda.synchronize()
    for b in range(2):
        s = slice(302 * b, 302 * b + 302)
        want = oda.attention(f64(x["q"])[b:b + 1], f64(k)[s], f64(v)[s], oda.Scores(), 0, HALF_STEP["bf16"])
        close(x["o"][b:b + 1], want[0], want[2], "o")
    assert bool((k[:300] == k[302:602]).all()) and not bool((k[300:302] == k[602:604]).all())
