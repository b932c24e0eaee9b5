"""The paged key/value cache on the GPU: append and attention, element by element against the
fp64 oracle, and a run of both with attention over documents."""
import os
import re

import numpy as np
import pytest

import paper_2601_20595_amd as csg
from oracle import doc_attention as oda

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from attn_util import DEV, HALF_STEP, TINY, TORCH, close, f64, ints, normal, pointers

pytestmark = pytest.mark.gpu


def _table(rng, lengths, page, spare=2, shared=()):
    """(page table, pages): pages in mixed order; shared (b0, b1, tokens): the first sequence's pages."""
    need = [max(1, -(-x // page)) for x in lengths]
    n = sum(need) + spare
    order = rng.permutation(n)
    t = np.full((len(need), max(need) + 1), -1, dtype=np.int32)  # behind the end: no page
    at = 0
    for b, x in enumerate(need):
        t[b, :x] = order[at:at + x]
        at += x
    for b0, b1, tokens in shared:
        t[b0:b1, :tokens // page] = t[b0, :tokens // page]
    return t, n


# sequences' new tokens, lengths after them, heads, key/value heads, head_dim, page size, rotated, interleaved
APPEND = {
    "one token": ([1], [1], 4, 2, 128, 16, 128, False),
    "decode": ([1] * 9, [1, 16, 17, 33, 100, 64, 65, 5, 2], 32, 8, 128, 16, 128, False),
    "far positions": ([1, 2], [1000001, 3000000], 2, 1, 64, 256, 64, False),
    "ragged, some without": ([0, 40, 0, 1, 33, 0], [7, 50, 0, 64, 33, 12], 6, 3, 64, 32, 32, True),
    "interleaved": ([17, 90], [17, 300], 5, 5, 128, 64, 128, True),
    "part of a head": ([50], [51], 3, 1, 128, 16, 48, False),
    "nothing rotated": ([20, 3], [30, 4], 4, 4, 64, 128, 0, False),
}


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", APPEND)
def test_append(name, dtype):
    new, lens, H, Hkv, D, page, rot, pairs = APPEND[name]
    rng = np.random.default_rng(3)
    n, tail = sum(new), 3
    if name == "far positions":  # only the last pages exist
        width = max(-(-x // page) for x in lens)
        table, pages = np.full((len(lens), width), -1, dtype=np.int32), 4
        for b, x in enumerate(lens):
            table[b, (x - 1) // page], table[b, (x - 2) // page] = 2 * b, 2 * b + (((x - 1) // page) != ((x - 2) // page))
    else:
        table, pages = _table(rng, lens, page)
    k, k64 = normal(1, (n + tail, Hkv, D), dtype)
    v, v64 = normal(2, (n + tail, Hkv, D), dtype)
    q, q64 = normal(3, (n + tail, H, D), dtype)
    kp, kp64 = normal(4, (pages, Hkv, page, D), dtype)
    vp, vp64 = normal(5, (pages, Hkv, page, D), dtype)
    freq = 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    pos = np.concatenate([np.arange(x - a, x) for a, x in zip(new, lens)]) if n else np.zeros(0, dtype=int)
    seq = np.repeat(np.arange(len(new)), new)
    kr, qr = oda.rotate(k64[:n], pos, freq, pairs), oda.rotate(q64[:n], pos, freq, pairs)
    at = (table[seq, pos // page], slice(None), pos % page)
    u = HALF_STEP[dtype]
    # a rounding of the result; fp32 products and the hardware's sine (2^-18 of a pair's size, which is
    # no more than the two values' sum)
    def bound(x, y):
        return u * np.abs(x) + 2.0 ** -17 * np.abs(y).max() + (TINY[dtype] if rot else 0)
    kp64[at], vp64[at] = kr, v64[:n]
    ek = np.zeros_like(kp64)
    ek[at] = bound(kr, k64[:n]) if rot else 0
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    dk, dv = kp.to(DEV), vp.to(DEV)
    out = torch.full((n + tail, H, D), 17.0, dtype=TORCH[dtype], device=DEV)
    c = csg.PagedCache(H, Hkv, D, dtype, pages, page, len(new), table.shape[1])
    inv = torch.tensor(freq, device=DEV) if rot else None
    # the projection's output: queries, keys and values of a token behind each other
    x = torch.cat([q, k, v], dim=1).to(DEV)
    torch.cuda.synchronize()
    c.append(dk, dv, x[:, H:H + Hkv], x[:, H + Hkv:], ints(pointers(new)), ints(lens), torch.tensor(table, device=DEV),
             inv_freq=inv, interleaved=pairs, q=x[:, :H], q_out=out, status=st)
    torch.cuda.synchronize()
    assert int(st) == 0
    close(dk, kp64, ek, "keys")
    close(dv, vp64, np.zeros_like(vp64), "values")
    close(out[:n], qr, bound(qr, q64[:n]) if rot else np.zeros_like(qr), "queries")
    assert bool((out[n:] == 17.0).all())


def test_append_without_queries_and_bad_pages():
    H, Hkv, D, page = 4, 2, 64, 16
    new, lens = [1, 1, 1, 2], [3, 20, 100, 1]
    table = np.array([[0, -1], [1, 99], [2, 3], [4, 5]], dtype=np.int32)
    k, _ = normal(1, (5, Hkv, D), "bf16")
    v, _ = normal(2, (5, Hkv, D), "bf16")
    kp, vp = (torch.full((6, Hkv, page, D), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    c = csg.PagedCache(H, Hkv, D, "bf16", 6, page, 4, 2)
    c.append(kp, vp, k.to(DEV), v.to(DEV), ints(pointers(new)), ints(lens), torch.tensor(table, device=DEV), status=st)
    torch.cuda.synchronize()
    # written: sequence 0's token at 2, sequence 3's at 0; page 99, position 99 of 32 and position -1 are not
    assert int(st) == 3
    want_k, want_v = torch.full_like(kp, 9.0), torch.full_like(vp, 9.0)
    for w, x in ((want_k, k), (want_v, v)):
        w[0, :, 2], w[4, :, 0] = x[0].to(DEV), x[4].to(DEV)
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)


# new tokens, lengths, heads, key/value heads, head_dim, page size, groups (b0, b1, shared tokens), cap, bias
ATTN = {
    "one key": ([1], [1], 4, 2, 128, 16, [], 0.0, False),
    "one sequence": ([1], [900], 32, 8, 128, 64, [], 0.0, False),
    "block edges": ([1] * 8, [31, 32, 33, 63, 64, 65, 127, 129], 8, 2, 64, 16, [], 0.0, False),
    "ragged new tokens": ([0, 5, 1, 40, 0, 3], [10, 5, 300, 90, 0, 77], 12, 4, 128, 32, [], 0.0, False),
    "many rows a head": ([7, 33], [200, 33], 10, 1, 64, 128, [], 0.0, False),
    "a group": ([1] * 6, [210, 257, 192, 300, 193, 1000], 8, 2, 128, 64, [(0, 6, 192)], 0.0, False),
    "groups between others": ([1, 2, 1, 3, 1, 1, 1], [40, 170, 161, 400, 33, 64, 65], 12, 4, 64, 16,
                              [(1, 4, 144), (4, 7, 32)], 0.0, False),
    "a prefix inside a block": ([1, 1, 2], [90, 59, 300], 4, 1, 128, 16, [(0, 3, 48)], 0.0, False),
    "a group with an empty suffix": ([1, 1], [64, 100], 4, 1, 128, 16, [(0, 2, 64)], 0.0, False),
    "cap": ([1, 4], [333, 70], 8, 2, 128, 256, [], 6.0, False),
    "bias": ([1, 3, 1], [200, 97, 130], 8, 4, 64, 16, [(0, 3, 80)], 0.0, True),
    "cap and bias": ([2] * 5, [400, 30, 260, 64, 129], 5, 5, 128, 32, [], 10.0, True),
    "groups of many sequences": ([1] * 300, [60 + (37 * i) % 90 for i in range(300)], 4, 2, 64, 16, [(0, 150, 48), (150, 300, 32)],
                                 0.0, False),
    "an empty group": ([1] * 5, [100, 90, 120, 80, 33], 4, 1, 64, 16, [(1, 3, 64), (3, 3, 32), (3, 5, 16)], 0.0, False),
    "many sequences": ([1] * 300, [1 + (37 * i) % 90 for i in range(300)], 4, 2, 64, 16, [], 0.0, False),
}


def _attn_case(name, dtype, sharp=1.0, stream=None):
    new, lens, H, Hkv, D, page, groups, cap, bias = ATTN[name]
    rng = np.random.default_rng(7)
    n, tail = sum(new), 2
    table, pages = _table(rng, lens, page, shared=groups)
    q, q64 = normal(1, (n + tail, H, D), dtype, sharp)
    kp, _ = normal(2, (pages, Hkv, page, D), dtype)
    vp, _ = normal(3, (pages, Hkv, page, D), dtype)
    kp64, vp64 = kp.double().numpy().copy(), vp.double().numpy().copy()
    # rows of a page that no sequence has hold NaN
    used = np.zeros((pages, page), dtype=bool)
    for b, x in enumerate(lens):
        i = np.arange(x)
        used[table[b][i // page], i % page] = True
    kp, vp = kp.clone(), vp.clone()
    for t in (kp, vp):
        t.permute(0, 2, 1, 3)[torch.tensor(~used)] = float("nan")
    slopes = (2.0 ** -np.arange(1, H + 1)).astype(np.float32) if bias else None
    sc = oda.Scores(None, cap, slopes, True)
    ptr = pointers(new)
    want = [np.zeros((n, H, D)), np.zeros((H, n)), np.zeros((n, H, D)), np.zeros((H, n))]
    for b, x in enumerate(lens):
        r = slice(ptr[b], ptr[b + 1])
        got = oda.attention(q64[r], oda.cached_rows(kp64, table[b], x), oda.cached_rows(vp64, table[b], x), sc, 0,
                            HALF_STEP[dtype], TINY[dtype])
        want[0][r], want[1][:, r], want[2][r], want[3][:, r] = got
    c = csg.PagedCache(H, Hkv, D, dtype, pages, page, len(new), table.shape[1])
    o = torch.full((n + tail, H, D), 17.0, dtype=TORCH[dtype], device=DEV)
    lse = torch.full((H, n + tail), 17.0, device=DEV)
    ws = torch.full((c.workspace_bytes(n + tail, len(groups)),), 255, dtype=torch.uint8, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    args = {"status": st, "softcap": cap, "stream": stream}
    if groups:
        # (groups are neighbours: the sequences between two groups would be one of their own)
        args["group_ptr"] = ints([g[0] for g in groups] + [groups[-1][1]])
        args["prefix"] = ints([g[2] for g in groups])
    if bias:
        args["slopes"] = torch.tensor(slopes, device=DEV)
    dev = [q.to(DEV), kp.to(DEV), vp.to(DEV), ints(ptr), ints(lens), torch.tensor(table, device=DEV)]
    torch.cuda.synchronize()
    c.attn(*dev, o, lse, ws, **args)
    torch.cuda.synchronize()
    assert int(st) == 0
    close(o[:n], want[0], want[2], "o")
    close(lse[:, :n], want[1], want[3], "lse")
    assert bool((o[n:] == 17.0).all()) and bool((lse[:, n:] == 17.0).all())
    return o, lse


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", ATTN)
def test_attention(name, dtype):
    _attn_case(name, dtype)


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("D,shared", [(64, 23), (128, 48), (128, 87)])
def test_a_groups_tokens_are_read_from_its_first_sequence(D, shared, new):
    """The others have no pages for them, and NaN where such a token would share a page with later ones."""
    H, Hkv, page, lens = 8, 2, 16, [200, 130, 150]
    rng = np.random.default_rng(5)
    table, pages = _table(rng, lens, page)
    kp, vp = (normal(s, (pages, Hkv, page, D), "bf16")[0] for s in (1, 2))
    for b in (1, 2):
        x = np.arange(shared)
        for t in (kp, vp):
            t[table[b][x // page], :, x % page] = t[table[0][x // page], :, x % page]
    q = normal(3, (3 * new, H, D), "bf16")[0].to(DEV)
    c = csg.PagedCache(H, Hkv, D, "bf16", pages, page, 3, table.shape[1])
    ws = torch.zeros(c.workspace_bytes(3 * new, 1), dtype=torch.uint8, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = []
    for gone in (False, True):
        if gone:
            for b in (1, 2):
                x = np.arange(shared)
                for t in (kp, vp):
                    t[table[b][x // page], :, x % page] = float("nan")
                table[b, :shared // page] = -1
        o, lse = torch.zeros_like(q), torch.zeros((H, 3 * new), device=DEV)
        c.attn(q, kp.to(DEV), vp.to(DEV), ints(pointers([new] * 3)), ints(lens), torch.tensor(table, device=DEV), o, lse, ws,
               group_ptr=ints([0, 3]), prefix=ints([shared]), status=st)
        torch.cuda.synchronize()
        out.append((o, lse))
    assert int(st) == 0
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


@pytest.mark.parametrize("new", [1, 40])
def test_long_runs(new):
    """So many keys a workgroup that it asks for pages again (narrow tasks: after 32 blocks of a wave;
    wide ones: after 64 steps), against fp64 on the GPU."""
    H, D, page, n = 128, 64, 64, 20000
    rng = np.random.default_rng(11)
    table, pages = _table(rng, [n], page)
    tab = torch.tensor(table, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    kp, vp = (torch.randn((pages, H, page, D), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    x = torch.randn((new, H + 3, D), generator=g, device=DEV).to(torch.bfloat16)
    q = x[:, 1:H + 1]  # a part of a wider tensor
    c = csg.PagedCache(H, H, D, "bf16", pages, page, 1, table.shape[1])
    o, ws = torch.empty((new, H, D), dtype=torch.bfloat16, device=DEV), torch.empty(c.workspace_bytes(new), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    c.attn(q, kp, vp, ints([0, new]), ints([n]), tab, o, None, ws)  # (no log-sum-exp wanted)
    torch.cuda.synchronize()
    at = torch.arange(n, device=DEV)
    place = tab[0].long()[at // page]
    u = HALF_STEP["bf16"]
    for h in range(0, H, 9):
        k, v, qh = kp[place, h, at % page].double(), vp[place, h, at % page].double(), q[:, h].double()
        s = (qh @ k.t()) * D ** -0.5
        s[at[None] > n - new + torch.arange(new, device=DEV)[:, None]] = float("-inf")
        p = torch.softmax(s, dim=1)
        want = p @ v
        # the oracle's bounds: a rounding of the output and of every weight, and 2^-17 of the scores' size
        size = (qh.abs() @ k.abs().t()) * D ** -0.5 + s.abs().nan_to_num(posinf=0.0) + 1.0
        bound = u * want.abs() + (p * (2 * 2.0 ** -17 * size + u)) @ v.abs()
        assert bool(((o[:, h].double() - want).abs() <= bound).all()), h


def test_sharp_scores_other_stream_same_bits():
    st = torch.cuda.Stream(device=DEV)
    one = _attn_case("groups between others", "f16", 5.0, st)
    two = _attn_case("groups between others", "f16", 5.0)
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])


def test_far_pages():
    """Pages beyond 2^32 elements of a cache, bit for bit as near ones."""
    H, Hkv, D, page, n = 16, 8, 128, 256, 700
    x = normal(1, (n, H + 2 * Hkv, D), "bf16")[0].to(DEV)
    out = []
    for pages in (3, 18000):
        kp, vp = (torch.empty((pages, Hkv, page, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        c = csg.PagedCache(H, Hkv, D, "bf16", pages, page, 1, 3)
        tab, ptr, lens = ints([[pages - 1, 0, pages - 2]]), ints([0, n]), ints([n])
        o, lse = torch.zeros((n, H, D), dtype=torch.bfloat16, device=DEV), torch.zeros((H, n), device=DEV)
        ws = torch.zeros(c.workspace_bytes(n), dtype=torch.uint8, device=DEV)
        c.append(kp, vp, x[:, H:H + Hkv], x[:, H + Hkv:], ptr, lens, tab)
        c.attn(x[:, :H], kp, vp, ptr, lens, tab, o, lse, ws)
        torch.cuda.synchronize()
        last = n - 2 * page
        out.append((o, lse, kp[-1].clone(), vp[-1].clone(), kp[-2, :, :last].clone()))
    for one, two in zip(*out):
        assert torch.equal(one, two)


def test_bad_pages_and_lengths_touch_nothing_else():
    H, Hkv, D, page = 4, 2, 64, 16
    lens = [40, 40, 1000, -3]
    table = np.array([[0, 1, 2], [3, -7, 1 << 30], [6, 7, 0], [1, 1, 1]], dtype=np.int32)
    kp, _ = normal(2, (8, Hkv, page, D), "bf16")
    vp, vp64 = normal(3, (8, Hkv, page, D), "bf16")
    q, q64 = normal(1, (4, H, D), "bf16")
    c = csg.PagedCache(H, Hkv, D, "bf16", 8, page, 4, 3)
    o, lse = torch.zeros((4, H, D), dtype=torch.bfloat16, device=DEV), torch.zeros((H, 4), device=DEV)
    ws = torch.zeros(c.workspace_bytes(4), dtype=torch.uint8, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    c.attn(q.to(DEV), kp.to(DEV), vp.to(DEV), ints([0, 1, 2, 3, 4]), ints(lens), torch.tensor(table, device=DEV), o, lse, ws, status=st)
    torch.cuda.synchronize()
    assert int(st) == 3
    k0, v0 = (oda.cached_rows(x.double().numpy(), table[0], 40) for x in (kp, vp))
    want = oda.attention(q64[:1], k0, v0, oda.Scores(), 0, HALF_STEP["bf16"])
    close(o[:1], want[0], want[2], "the good sequence")
    assert bool((o[3] == 0).all()) and bool((lse[:, 3] == float("-inf")).all())


def test_more_new_tokens_than_the_sequence_has():
    H, D, page = 2, 64, 16
    kp, _ = normal(2, (2, 1, page, D), "bf16")
    q, _ = normal(1, (5, H, D), "bf16")
    c = csg.PagedCache(H, 1, D, "bf16", 2, page, 1, 2)
    ws = torch.zeros(c.workspace_bytes(5), dtype=torch.uint8, device=DEV)
    for n, bits in ((5, 0), (4, 2)):
        o = torch.zeros((5, H, D), dtype=torch.bfloat16, device=DEV)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        c.attn(q.to(DEV), kp.to(DEV), kp.to(DEV), ints([0, 5]), ints([n]), ints([[0, 1]]), o, None, ws, status=st)
        torch.cuda.synchronize()
        assert int(st) == bits


def test_captured_and_replayed():
    """A decode step (append, attention) as one graph, replayed as the sequences grow."""
    H, Hkv, D, page, batch = 8, 2, 128, 16, 5
    rng = np.random.default_rng(1)
    table, pages = _table(rng, [200] * batch, page)
    c = csg.PagedCache(H, Hkv, D, "bf16", pages, page, batch, table.shape[1])
    kp, vp = (normal(s, (pages, Hkv, page, D), "bf16")[0].to(DEV) for s in (1, 2))
    x = torch.zeros((batch, H + 2 * Hkv, D), dtype=torch.bfloat16, device=DEV)
    qo, o = (torch.zeros((batch, H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lse = torch.zeros((H, batch), device=DEV)
    ws = torch.zeros(c.workspace_bytes(batch), dtype=torch.uint8, device=DEV)
    ptr, lens, tab = ints(range(batch + 1)), ints([1] * batch), torch.tensor(table, device=DEV)
    inv = torch.tensor(10000.0 ** (-np.arange(0, D, 2) / D), device=DEV)

    def step(stream):
        c.append(kp, vp, x[:, H:H + Hkv], x[:, H + Hkv:], ptr, lens, tab, inv_freq=inv, q=x[:, :H], q_out=qo, stream=stream)
        c.attn(qo, kp, vp, ptr, lens, tab, o, lse, ws, stream=stream)

    st = torch.cuda.Stream(device=DEV)
    step(st)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        step(st)
    for t, lengths in enumerate(([1, 15, 16, 17, 100], [2, 16, 17, 18, 101], [180, 3, 64, 65, 1])):
        x.copy_(normal(20 + t, tuple(x.shape), "bf16")[0])
        lens.copy_(ints(lengths))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = [y.clone() for y in (kp, vp, o, lse)]
        step(None)
        torch.cuda.synchronize()
        for one, two in zip(got, (kp, vp, o, lse)):
            assert torch.equal(one, two)


def test_prompt_drafts_and_decoding_agree_with_documents():
    """A run as a model makes it: two prompts through attention over documents, their keys into the
    cache; then tokens one by one and as drafts, against documents of the whole text."""
    H, Hkv, D, page, dtype = 8, 2, 128, 16, "bf16"
    prompt, total = [70, 33], [90, 45]
    rng = np.random.default_rng(2)
    table, pages = _table(rng, total, page)
    inv = 10000.0 ** (-np.arange(0, D, 2) / D)
    x = [normal(3 + b, (total[b], H + 2 * Hkv, D), dtype) for b in range(2)]
    c = csg.PagedCache(H, Hkv, D, dtype, pages, page, 2, table.shape[1])
    a = csg.DocAttn(H, Hkv, D, dtype)
    kp, vp = (torch.full((pages, Hkv, page, D), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    tab, freq = torch.tensor(table, device=DEV), torch.tensor(inv, device=DEV)
    u = HALF_STEP[dtype]
    want = []
    for b in range(2):
        y = x[b][1]
        pos = np.arange(total[b])

        def rounded(z):  # the cache holds rounded keys
            return torch.tensor(z).to(TORCH[dtype]).double().numpy()

        q, k = rounded(oda.rotate(y[:, :H], pos, inv, False)), rounded(oda.rotate(y[:, H:H + Hkv], pos, inv, False))
        want.append((q, k) + oda.attention(q, k, y[:, H + Hkv:], oda.Scores(), 0, u))
    at = [0, 0]
    for new in (prompt, [1, 1], [4, 0], [1, 3], [14, 8]):
        n = sum(new)
        rows = [slice(s, s + d) for s, d in zip(at, new)]
        at = [s + d for s, d in zip(at, new)]
        y = torch.cat([x[b][0][rows[b]] for b in range(2)]).to(DEV)
        q, o, o2 = (torch.empty((n, H, D), dtype=TORCH[dtype], device=DEV) for _ in range(3))
        lse, lse2 = torch.empty((H, n), device=DEV), torch.empty((H, n), device=DEV)
        ws = torch.empty(c.workspace_bytes(n), dtype=torch.uint8, device=DEV)
        ptr, lens = ints(pointers(new)), ints(at)
        c.append(kp, vp, y[:, H:H + Hkv], y[:, H + Hkv:], ptr, lens, tab, inv_freq=freq, q=y[:, :H], q_out=q)
        c.attn(q, kp, vp, ptr, lens, tab, o, lse, ws)
        keys = [torch.tensor(oda.cached_rows(np.arange(pages * page).reshape(pages, 1, page, 1), table[b], at[b])[:, 0, 0], device=DEV)
                for b in range(2)]
        k, v = (torch.cat([z.permute(0, 2, 1, 3).reshape(pages * page, Hkv, D)[i] for i in keys]) for z in (kp, vp))
        a.forward(q, k, v, ptr, ints(pointers(at)), o2, lse2)
        torch.cuda.synchronize()
        # rotated keys and queries may each be off by a rounding: 2 u of the products' size each, twice
        # in a weight, on top of the bounds for exact inputs
        ref = [np.concatenate([want[b][i][rows[b]] for b in range(2)]) for i in (2, 4)]
        size = np.concatenate([(np.abs(want[b][0][rows[b]]).sum(-1) * np.abs(want[b][1]).max() / np.sqrt(D)) for b in range(2)])
        wide = ref[1] + (4 * u * size)[..., None] * np.abs(x[0][1]).max()
        close(o, ref[0], wide, "cache")
        close(o2, ref[0], wide, "documents")
        # the two see the same rounded keys: only the order of sums and of weights' references differs
        both = 2 * ref[1]
        close(o, f64(o2), both, "cache against documents")


def test_readme_example():
    """The attention example of README.md runs, and its cache gives what its documents give."""
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    blocks = re.findall(r"```py\n(.*?)```", text, re.S)
    assert len(blocks) == 1
    names = {}
    exec(compile(blocks[0], "README.md", "exec"), names)
    torch.cuda.synchronize()
    got = names["o"].clone()
    # the same rotated queries and keys as documents: the keys of a sequence from its pages
    pages, table, lens = names["k_pages"], names["table"].long(), names["lens"].tolist()
    k = torch.cat([pages[table[b]].permute(0, 2, 1, 3).reshape(-1, 8, 128)[:n] for b, n in enumerate(lens)])
    names["attn"].forward(names["q"], k, names["v"], names["ptr"], names["ptr"], names["o"], names["lse"])
    torch.cuda.synchronize()
    # a rounding of each of the two outputs and of their weights: values are averaged, |v| < 6
    assert float((got.float() - names["o"].float()).abs().max()) <= 4 * HALF_STEP["bf16"] * 6
    assert all(bool(torch.isfinite(names[x].float()).all()) for x in ("dq", "dk", "dv", "lse"))
