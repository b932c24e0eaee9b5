"""Attention over both paged caches where entries of the page table name no page: their keys and values are zeros,
whatever page 0 holds."""
import numpy as np
import pytest

import paper_2601_20595_amd as csg
from oracle import doc_attention as oda

from test_gpu_cache import _table

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from attn_util import DEV, HALF_STEP, TINY, TORCH, close, ints, normal, pointers
    from cache4_util import pages4

pytestmark = pytest.mark.gpu

# sequences' new tokens, lengths, heads, key/value heads, page size, groups (first, end, shared tokens), cap, bias
CALLS = {
    "few rows": ([1, 1, 1], [200, 70, 900], 8, 2, 16, [], 0.0, False),
    "few rows, a cap and a bias": ([1, 2, 0, 1], [700, 64, 9, 333], 8, 1, 64, [], 6.0, True),
    "one of many rows": ([40] + [1] * 20, [90] + [1 + 13 * i for i in range(20)], 8, 2, 16, [], 0.0, False),
    "a wave each": ([1] * 60, [3 + (i * i * 7) % 600 for i in range(60)], 16, 8, 16, [], 0.0, True),
    "some rows": ([3] * 5, [3, 65, 128, 500, 1100], 16, 2, 32, [], 0.0, False),
    "many rows": ([40, 70], [40, 1500], 8, 2, 16, [], 0.0, True),
    "groups": ([1, 9, 1, 2, 1], [300, 280, 400, 310, 90], 16, 2, 16, [(0, 2, 208), (2, 4, 256)], 0.0, False),
    "a wave each, beside groups": ([1] * 60, [160 + (i * 37) % 300 for i in range(60)], 32, 8, 16, [(0, 25, 128), (25, 60, 96)], 4.0, True),
}


@pytest.mark.parametrize("dtype, D", [("bf16", 128), ("bf16", 64), ("f16", 128), ("f16", 64)])
@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("bits", [16, 4])
def test_keys_without_a_page_are_zeros(bits, name, dtype, D):
    new, lens, H, Hkv, page, groups, cap, bias = CALLS[name]
    rng = np.random.default_rng(5)
    table, pages = _table(rng, lens, page, shared=groups)
    table, pages = np.where(table >= 0, table + 1, table).astype(np.int32), pages + 1  # (nobody has page 0)
    # about a third of the entries name no page, the first and the last of a sequence among them
    for b, x in enumerate(lens):
        held = -(-x // page)
        gone = rng.random(held) < 0.3
        gone[0] |= b % 3 == 0
        gone[-1] |= b % 4 == 1
        table[b, :held][gone] = rng.choice([-1, pages, 1 << 30, -(1 << 31)], int(gone.sum()))
    q, q64 = normal(1, (sum(new), H, D), dtype)
    if bits == 4:
        kp, kp64 = pages4(2, pages, Hkv, page, D, dtype)
        vp, vp64 = pages4(3, pages, Hkv, page, D, dtype)
        for p in (kp, vp):
            p[0] = 255  # (NaN, all of it)
        kind = csg.PagedCache4
    else:
        kp, kp64 = normal(2, (pages, Hkv, page, D), dtype)
        vp, vp64 = normal(3, (pages, Hkv, page, D), dtype)
        for p in (kp, vp):
            p[0] = float("nan")
        kind = csg.PagedCache
    from_first = table.copy()
    for b0, b1, shared in groups:
        from_first[b0:b1, :shared // page] = table[b0, :shared // page]
    rows = np.where((from_first >= 0) & (from_first < pages), from_first, pages)
    kp64, vp64 = (np.concatenate([x, np.zeros((1, Hkv, page, D))]) for x in (kp64, vp64))
    slopes = (2.0 ** -np.arange(1, H + 1)).astype(np.float32) if bias else None
    sc = oda.Scores(None, cap, slopes, True)
    ptr = pointers(new)
    c = kind(H, Hkv, D, dtype, pages, page, len(new), table.shape[1])
    o, lse = torch.full_like(q, 17.0, device=DEV), torch.full((H, len(q)), 17.0, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.full((c.workspace_bytes(len(q), len(groups)),), 255, dtype=torch.uint8, device=DEV)
    args = {"status": st, "softcap": cap}
    if groups:
        args["group_ptr"] = ints([g[0] for g in groups] + [groups[-1][1]])
        args["prefix"] = ints([g[2] for g in groups])
    if bias:
        args["slopes"] = torch.tensor(slopes, device=DEV)
    c.attn(q.to(DEV), kp.to(DEV), vp.to(DEV), ints(ptr), ints(lens), torch.tensor(table, device=DEV), o, lse, ws, **args)
    torch.cuda.synchronize()
    assert int(st) == 1
    want = [np.zeros((len(q), H, D)), np.zeros((H, len(q))), np.zeros((len(q), H, D)), np.zeros((H, len(q)))]
    for b, x in enumerate(lens):
        r = slice(ptr[b], ptr[b + 1])
        k, v = (oda.cached_rows(y, rows[b], x) for y in (kp64, vp64))
        want[0][r], want[1][:, r], want[2][r], want[3][:, r] = oda.attention(q64[r], k, v, sc, 0, HALF_STEP[dtype], TINY[dtype])
    close(o, want[0], want[2], "o")
    close(lse, want[1], want[3], "lse")
