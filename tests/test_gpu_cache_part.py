"""Calls of the paged cache on a part of a batch's rows: pointers that begin behind row 0."""
import numpy as np
import pytest

import paper_2601_20595_amd as csg
from oracle import doc_attention as oda

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from attn_util import DEV, HALF_STEP, TINY, TORCH, close, ints, normal, pointers

pytestmark = pytest.mark.gpu

# new tokens, lengths; the part is sequences first .. last - 1
BATCHES = {
    "decode": ([1] * 6, [20, 33, 17, 64, 5, 90], 2, 5),
    "prompts, then single tokens": ([30, 45, 1, 1, 1], [30, 60, 100, 40, 33], 2, 5),
    "prompts of a mixed batch": ([1, 1, 40, 25, 1], [50, 20, 70, 25, 9], 2, 4),
    "the first has no tokens": ([3, 0, 2, 1], [30, 12, 20, 7], 1, 4),
}
H, HKV, D, PAGE = 8, 2, 128, 16


def _batch(name, dtype):
    new, lens, first, last = BATCHES[name]
    need = [-(-x // PAGE) for x in lens]
    table = np.full((len(new), max(need)), -1, dtype=np.int32)
    order = np.random.default_rng(3).permutation(sum(need))
    for b, x in enumerate(need):
        table[b, :x], order = order[:x], order[x:]
    n = sum(new)
    x = normal(1, (n, H + 2 * HKV, D), dtype)[0]
    pages = [normal(i, (sum(need), HKV, PAGE, D), dtype)[0].to(DEV) for i in (2, 3)]
    return new, lens, first, last, table, x, pages


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", BATCHES)
def test_append(name, dtype):
    new, lens, first, last, table, x, (kp, vp) = _batch(name, dtype)
    n, ptr = sum(new), pointers(new)
    x = x.to(DEV)
    freq = torch.tensor(10000.0 ** (-np.arange(0, D, 2) / D), device=DEV)

    def append(lo, hi, kp, vp, out):
        c = csg.PagedCache(H, HKV, D, dtype, kp.shape[0], PAGE, hi - lo, table.shape[1])
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        c.append(kp, vp, x[:, H:H + HKV], x[:, H + HKV:], ints(ptr)[lo:hi + 1], ints(lens)[lo:hi], torch.tensor(table[lo:hi], device=DEV),
                 inv_freq=freq, q=x[:, :H], q_out=out, status=st)
        torch.cuda.synchronize()
        assert int(st) == 0

    all_k, all_v, part_k, part_v = kp.clone(), vp.clone(), kp.clone(), vp.clone()
    all_q, part_q = (torch.full((n, H, D), 17.0, dtype=TORCH[dtype], device=DEV) for _ in range(2))
    append(0, len(new), all_k, all_v, all_q)
    append(first, last, part_k, part_v, part_q)
    # the part's tokens as in the whole batch's call, everything else as it was
    want_k, want_v = kp.clone(), vp.clone()
    for b in range(first, last):
        at = np.arange(lens[b] - new[b], lens[b])
        page, row = torch.tensor(table[b, at // PAGE]).long().to(DEV), torch.tensor(at % PAGE).to(DEV)
        want_k[page, :, row], want_v[page, :, row] = all_k[page, :, row], all_v[page, :, row]
    assert torch.equal(part_k, want_k) and torch.equal(part_v, want_v)
    r = slice(ptr[first], ptr[last])
    assert torch.equal(part_q[r], all_q[r])
    assert bool((part_q[:r.start] == 17.0).all()) and bool((part_q[r.stop:] == 17.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", BATCHES)
def test_attention(name, dtype):
    new, lens, first, last, table, x, (kp, vp) = _batch(name, dtype)
    n, ptr = sum(new), pointers(new)
    q64 = x[:, :H].double().numpy()
    c = csg.PagedCache(H, HKV, D, dtype, kp.shape[0], PAGE, last - first, table.shape[1])
    o, lse = torch.full((n, H, D), 17.0, dtype=TORCH[dtype], device=DEV), torch.full((H, n), 17.0, device=DEV)
    ws = torch.full((c.workspace_bytes(n),), 255, dtype=torch.uint8, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    c.attn(x.to(DEV)[:, :H], kp, vp, ints(ptr)[first:last + 1], ints(lens)[first:last], torch.tensor(table[first:last], device=DEV),
           o, lse, ws, status=st)
    torch.cuda.synchronize()
    assert int(st) == 0
    k64, v64 = kp.cpu().double().numpy(), vp.cpu().double().numpy()
    for b in range(first, last):
        r = slice(ptr[b], ptr[b + 1])
        want = oda.attention(q64[r], oda.cached_rows(k64, table[b], lens[b]), oda.cached_rows(v64, table[b], lens[b]), oda.Scores(), 0,
                             HALF_STEP[dtype], TINY[dtype])
        close(o[r], want[0], want[2], "o")
        close(lse[:, r], want[1], want[3], "lse")
    r = slice(ptr[first], ptr[last])
    for rows in (slice(0, r.start), slice(r.stop, n)):
        assert bool((o[rows] == 17.0).all()) and bool((lse[:, rows] == 17.0).all())
