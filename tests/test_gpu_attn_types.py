"""Each argument of the attention calls with elements of another type is refused by its name."""
import pytest

import paper_2601_20595_amd as csg

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from attn_util import DEV, ints

pytestmark = pytest.mark.gpu

H, HKV, D, N = 4, 2, 64, 3
OTHER = {torch.bfloat16: torch.float16, torch.int32: torch.float32, torch.float32: torch.int32, torch.float64: torch.int64}


def _refuses_each(call, args):
    call(**args)
    torch.cuda.synchronize()
    for name, t in args.items():
        if not torch.is_tensor(t) or t.dtype not in OTHER:
            continue
        with pytest.raises(ValueError, match="^%s must be " % name):
            call(**{**args, name: t.to(OTHER[t.dtype])})


def _heads(heads):
    return torch.zeros((N, heads, D), dtype=torch.bfloat16, device=DEV)


def test_documents():
    a = csg.DocAttn(H, HKV, D, "bf16")
    args = dict(q=_heads(H), k=_heads(HKV), v=_heads(HKV), q_ptr=ints([0, N]), k_ptr=ints([0, N]), o=_heads(H),
                lse=torch.zeros((H, N), device=DEV), prefix=ints([1]), slopes=torch.zeros(H, device=DEV))
    _refuses_each(a.forward, args)
    args.update(d_o=_heads(H), dq=_heads(H), dk=_heads(HKV), dv=_heads(HKV),
                workspace=torch.zeros(a.workspace_bytes(N, N), dtype=torch.uint8, device=DEV))
    _refuses_each(a.backward, args)


def test_cache():
    c = csg.PagedCache(H, HKV, D, "bf16", 2, 16, 1, 2)
    pages = [torch.zeros((2, HKV, 16, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    args = dict(k_pages=pages[0], v_pages=pages[1], k=_heads(HKV), v=_heads(HKV), q_ptr=ints([0, N]), lens=ints([5]),
                page_table=ints([[0, 1]]), inv_freq=torch.zeros(D // 2, dtype=torch.float64, device=DEV), q=_heads(H), q_out=_heads(H),
                status=ints([0]))
    _refuses_each(c.append, args)
    args = dict(q=_heads(H), k_pages=pages[0], v_pages=pages[1], q_ptr=ints([0, N]), lens=ints([5]), page_table=ints([[0, 1]]),
                o=_heads(H), lse=torch.zeros((H, N), device=DEV), workspace=torch.zeros(c.workspace_bytes(N, 1), dtype=torch.uint8, device=DEV),
                group_ptr=ints([0, 1]), prefix=ints([2]), slopes=torch.zeros(H, device=DEV), status=ints([0]))
    _refuses_each(c.attn, args)


def test_queries_and_their_output_go_together():
    c = csg.PagedCache(H, HKV, D, "bf16", 2, 16, 1, 2)
    pages = [torch.zeros((2, HKV, 16, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for p in ({"q": _heads(H)}, {"q_out": _heads(H)}):
        with pytest.raises(csg.CsgError, match="go together"):
            c.append(*pages, _heads(HKV), _heads(HKV), ints([0, N]), ints([5]), ints([[0, 1]]), **p)
