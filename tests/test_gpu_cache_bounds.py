"""Bounds of the paged cache that do not ascend: nothing outside is touched, and where they name
more rows than there are the status says so."""
import numpy as np
import pytest

import paper_2601_20595_amd as csg

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from attn_util import DEV, ints, normal

pytestmark = pytest.mark.gpu

H, HKV, D, PAGE, N = 32, 1, 64, 16, 8


@pytest.mark.parametrize("ptr, groups, bit", [([0, 8, 0, 8, 0, 8, 0], None, 2), ([0, 8, -5, 100, 0, 8, 8], None, 2),
                                              ([0, 2, 4, 6, 7, 8, 8], [0, 6, 0, 6, 0, 6, 0], 2), ([0, 3, 2, 6, 7, 8, 8], None, 0)])
def test_bounds_that_do_not_ascend(ptr, groups, bit):
    batch = len(ptr) - 1
    table = np.arange(batch * 4, dtype=np.int32).reshape(batch, 4)
    kp, vp = (normal(i, (batch * 4, HKV, PAGE, D), "bf16")[0].to(DEV) for i in (1, 2))
    q = normal(3, (N, H, D), "bf16")[0].to(DEV)
    k0, v0 = kp.clone(), vp.clone()
    c = csg.PagedCache(H, HKV, D, "bf16", batch * 4, PAGE, batch, 4)
    n_groups = 0 if groups is None else len(groups) - 1
    need, guard = c.workspace_bytes(N, n_groups), 1 << 16
    ws = torch.full((need + guard,), 170, dtype=torch.uint8, device=DEV)
    o = torch.full((N + 4, H, D), 17.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((H * N + 64,), 17.0, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    p = {} if groups is None else {"group_ptr": ints(groups), "prefix": ints([20] * n_groups)}
    c.attn(q, kp, vp, ints(ptr), ints([60] * batch), torch.tensor(table, device=DEV), o[:N], lse[:H * N], ws[:need], status=st, **p)
    torch.cuda.synchronize()
    assert int(st) == bit
    assert torch.equal(kp, k0) and torch.equal(vp, v0)
    assert bool((ws[need:] == 170).all()) and bool((o[N:] == 17.0).all()) and bool((lse[H * N:] == 17.0).all())
