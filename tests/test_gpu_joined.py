"""Results over disjoint keys joined by their log-sum-exp, and the gradients of such results: two
calls over documents, and ring attention with one."""
import numpy as np
import pytest

import paper_2601_20595_amd as csg
from grad_norms import check_norm, gradient_errors
from oracle import doc_attention as oda

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from attn_util import DEV, HALF_STEP, TINY, TORCH, close, f64, ints, normal, pointers

pytestmark = pytest.mark.gpu


def _join(parts, dtype):
    """o and lse of all keys from each part's, in fp32, the output rounded once more."""
    lse = torch.logsumexp(torch.stack([x[1] for x in parts]), dim=0)
    o = sum(x[0].float() * torch.exp(x[1] - lse).t()[..., None] for x in parts)
    return o.to(TORCH[dtype]), lse


def _joined_gradients(a, q, do, o, lse, parts):
    """Each part's gradients from the joined output: (dq of each, dk of each, dv of each)."""
    n, out = q.shape[0], []
    qp = ints([0, n])
    for k, v in parts:
        d = [torch.empty_like(t) for t in (q, k, v)]
        ws = torch.empty(a.workspace_bytes(n, k.shape[0]), dtype=torch.uint8, device=DEV)
        a.backward(q, k, v, qp, ints([0, k.shape[0]]), o, lse, do, *d, ws, joined=True)
        out.append([f64(t) for t in d])
    torch.cuda.synchronize()
    return list(zip(*out))


def _check_joined(x, sizes, got, dtype, row=0.0):
    """x: q, all keys, all values, do in fp64; sizes: the parts' keys; got: _joined_gradients."""
    p = pointers(sizes)
    want, error = gradient_errors(*x, oda.Scores(causal=False), 0, HALF_STEP[dtype], TINY[dtype],
                                  parts=[slice(a, b) for a, b in zip(p, p[1:])], row=row)
    rounded = sum((HALF_STEP[dtype] * y) ** 2 for y in got[0])  # each part's dq is rounded
    check_norm(sum(got[0]), want[0], np.sqrt(error[0] ** 2 + rounded), "dq")
    check_norm(np.concatenate(got[1]), want[1], error[1], "dk")
    check_norm(np.concatenate(got[2]), want[2], error[2], "dv")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
def test_joined_over_two_sets_of_keys(D, dtype):
    H, Hkv, n, sizes = 8, 2, 150, [200, 333]
    q, q64 = normal(1, (n, H, D), dtype, 3.0)
    k, k64 = normal(2, (sum(sizes), Hkv, D), dtype)
    v, v64 = normal(3, (sum(sizes), Hkv, D), dtype)
    do, do64 = normal(4, (n, H, D), dtype)
    q, do = q.to(DEV), do.to(DEV)
    sets = [(t[0].to(DEV).contiguous(), t[1].to(DEV).contiguous()) for t in zip(k.split(sizes), v.split(sizes))]
    a = csg.DocAttn(H, Hkv, D, dtype, causal=False)
    parts = []
    for kk, vv in sets:
        parts.append((torch.empty_like(q), torch.empty((H, n), device=DEV)))
        a.forward(q, kk, vv, ints([0, n]), ints([0, kk.shape[0]]), *parts[-1])
    o, lse = _join(parts, dtype)
    want, l64, bound, bl = oda.attention(q64, k64, v64, oda.Scores(causal=False), 0, HALF_STEP[dtype], TINY[dtype])
    # each part's output was rounded too: at most u |o| of its share, whose sizes the weights' bound covers
    close(o, want, 2 * bound, "o")
    close(lse, l64, 2 * bl, "lse")
    _check_joined((q64, k64, v64, do64), sizes, _joined_gradients(a, q, do, o, lse, sets), dtype)


def test_joined_with_ring_attention():
    """A rank's rows see the keys of two ranks by ring attention and 77 more by documents: output,
    log-sum-exp and gradients of all keys."""
    H, Hkv, D, n, shard, more = 8, 2, 128, 200, 256, 77
    m = 2 * shard + more
    q, q64 = normal(1, (n, H, D), "bf16", 2.0)
    k, k64 = normal(2, (m, Hkv, D), "bf16")
    v, v64 = normal(3, (m, Hkv, D), "bf16")
    do, do64 = normal(4, (n, H, D), "bf16")
    q, k, v, do = (t.to(DEV) for t in (q, k, v, do))
    plan = csg.AttnPlan(H, Hkv, D, n, csg.Schedule.uniform(2, 0, shard, 2, "ring"), cfg={"timeout_ms": 1000})
    kl, vl = k[:2 * shard].clone(), v[:2 * shard].clone()
    kl[shard:], vl[shard:] = 0, 0  # the other rank's rows arrive
    ring = torch.empty_like(q), torch.empty((H, n), device=DEV)
    compute, copy = torch.cuda.Stream(device=DEV), torch.cuda.Stream(device=DEV)
    torch.cuda.synchronize()
    plan.ring_attn(q, kl, vl, k[:2 * shard], v[:2 * shard], *ring, "overlap", compute, copy)
    plan.check()
    torch.cuda.synchronize()
    plan.close()
    a = csg.DocAttn(H, Hkv, D, "bf16", causal=False)
    rest = torch.empty_like(q), torch.empty((H, n), device=DEV)
    kr, vr = k[2 * shard:].contiguous(), v[2 * shard:].contiguous()
    a.forward(q, kr, vr, ints([0, n]), ints([0, more]), *rest)
    o, lse = _join([ring, rest], "bf16")
    want, l64, bound, bl = oda.attention(q64, k64, v64, oda.Scores(causal=False), 0, HALF_STEP["bf16"])
    close(o, want, 2 * bound, "o")
    # ring attention sums its weights after they are rounded: its sum is off by at most u of itself, and so
    # its share and the joined sum are
    u = HALF_STEP["bf16"]
    close(lse, l64, 2 * bl + u, "lse")
    _check_joined((q64, k64, v64, do64), [2 * shard, more], _joined_gradients(a, q, do, o, lse, [(kl, vl), (kr, vr)]), "bf16", row=u)
