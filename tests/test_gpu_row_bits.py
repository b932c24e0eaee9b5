"""A row's result is its own, bit for bit, whatever the other rows of its tile hold."""
import pytest

import paper_2601_20595_amd as csg

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from attn_util import DEV, ints, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
def test_documents_beside_a_row_of_enormous_scores(D):
    """Scores near fp32's largest number make a row's own reference move with every block of keys."""
    n, m = 32, 600
    q, k, v = (normal(i, (r, 1, D), "bf16")[0] for i, r in ((1, n), (2, m), (3, m)))
    k[..., 0] = torch.linspace(0.5, 1.0, m)[:, None].to(torch.bfloat16) * 1e19
    k[..., 1:] *= 3
    q[..., 0] = 0
    a = csg.DocAttn(1, 1, D, "bf16", causal=False)
    out = []
    for size in (0.0, 2e19):
        x = q.clone()
        x[5, 0, 0] = size
        o, lse = torch.zeros((n, 1, D), dtype=torch.bfloat16, device=DEV), torch.zeros((1, n), device=DEV)
        a.forward(x.to(DEV), k.to(DEV), v.to(DEV), ints([0, n]), ints([0, m]), o, lse)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(o.float()).all()) and bool(torch.isfinite(lse).all())
        out.append((torch.cat([o[:5], o[6:]]), torch.cat([lse[:, :5], lse[:, 6:]], dim=1)))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


def test_a_sequence_beside_one_of_enormous_scores():
    """Two sequences that share a prompt, their rows in one tile."""
    D, page, shared, lens = 128, 64, 320, [330, 340]
    kp, vp = (normal(i, (8, 1, page, D), "bf16")[0] for i in (1, 2))
    kp[..., 0] = torch.linspace(0.5, 1.0, 8 * page).view(8, 1, page).to(torch.bfloat16) * 1e19
    kp[..., 1:] *= 3
    table = torch.tensor([[0, 1, 2, 3, 4, 5], [0, 1, 2, 3, 4, 6]], dtype=torch.int32, device=DEV)
    q = normal(3, (2, 1, D), "bf16")[0]
    q[..., 0] = 0
    c = csg.PagedCache(1, 1, D, "bf16", 8, page, 2, 6)
    out = []
    for size in (0.0, 2e19):
        x = q.clone()
        x[1, 0, 0] = size
        o, lse = torch.zeros((2, 1, D), dtype=torch.bfloat16, device=DEV), torch.zeros((1, 2), device=DEV)
        ws = torch.zeros(c.workspace_bytes(2, 1), dtype=torch.uint8, device=DEV)
        c.attn(x.to(DEV), kp.to(DEV), vp.to(DEV), ints([0, 1, 2]), ints(lens), table, o, lse, ws, group_ptr=ints([0, 2]), prefix=ints([shared]))
        torch.cuda.synchronize()
        assert bool(torch.isfinite(o.float()).all()) and bool(torch.isfinite(lse).all())
        out.append((o[:1].clone(), lse[:, :1].clone()))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
