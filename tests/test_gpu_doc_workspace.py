"""Workspaces of the gradient of attention over packed documents on the GPU."""
import pytest

import paper_2601_20595_amd as csg

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from attn_util import DEV, ints, normal

pytestmark = pytest.mark.gpu


def test_a_workspace_of_more_rows_serves_fewer():
    """Fewer rows may be cut into more parts: the workspace made for the largest batch holds them."""
    H, D = 12, 64
    a = csg.DocAttn(H, H, D, "bf16")
    ws = torch.empty(a.workspace_bytes(6000, 6000), dtype=torch.uint8, device=DEV)
    for n in (6000, 4096, 1500, 300, 1):
        q, k, v, do = (normal(i, (n, H, D), "bf16")[0].to(DEV) for i in range(4))
        o, lse, p = torch.empty_like(q), torch.empty((H, n), device=DEV), ints([0, n])
        a.forward(q, k, v, p, p, o, lse)
        d = []
        for w in (ws, torch.empty(a.workspace_bytes(n, n), dtype=torch.uint8, device=DEV)):
            d.append([torch.zeros_like(t) for t in (q, k, v)])
            a.backward(q, k, v, p, p, o, lse, do, *d[-1], w)
        torch.cuda.synchronize()
        for one, two in zip(*d):
            assert torch.equal(one, two), n


def test_no_rows_need_no_workspace():
    H, Hkv, D, m = 8, 2, 128, 100
    a = csg.DocAttn(H, Hkv, D, "bf16")
    q, k, v = (normal(i, s, "bf16")[0].to(DEV) for i, s in enumerate(((0, H, D), (m, Hkv, D), (m, Hkv, D))))
    o, lse = torch.empty_like(q), torch.empty((H, 0), device=DEV)
    dq, dk, dv = (torch.full_like(t, 17.0) for t in (q, k, v))
    ws = torch.empty(a.workspace_bytes(0, m), dtype=torch.uint8, device=DEV)
    a.backward(q, k, v, ints([0, 0]), ints([0, m]), o, lse, torch.empty_like(q), dq, dk, dv, ws)
    torch.cuda.synchronize()
    assert bool((dk == 0).all()) and bool((dv == 0).all())
