"""Attention over packed documents and its gradient on the GPU, element by element against the
fp64 oracle with the bounds that it derives."""
import numpy as np
import pytest

import paper_2601_20595_amd as csg
from oracle import doc_attention as oda

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from attn_util import DEV, TORCH, close, doc_reference, f64, ints, normal, pointers

pytestmark = pytest.mark.gpu

# rows and keys of the documents, heads, key/value heads, head_dim, causal, prefixes, cap, bias
CASES = {
    "one row, one key": ([1], [1], 4, 4, 64, True, None, 0.0, False),
    "one row, many keys": ([1], [777], 4, 1, 128, True, None, 0.0, False),
    "tile and block edges": ([31, 32, 33, 64, 65], [31, 32, 33, 64, 65], 4, 1, 128, True, None, 0.0, False),
    "edges of 128": ([127, 128, 129, 1], [127, 128, 129, 1], 3, 3, 64, True, None, 0.0, False),
    "not causal": ([200, 5, 70], [130, 300, 70], 6, 3, 128, False, None, 0.0, False),
    "more rows than keys": ([100, 70, 9], [40, 1, 9], 8, 2, 64, True, None, 0.0, False),
    "empty documents": ([0, 60, 0, 0, 33, 0], [20, 0, 0, 15, 70, 0], 4, 2, 128, True, None, 0.0, False),
    "prefix": ([150, 90, 20, 64], [150, 200, 20, 10], 5, 1, 128, True, [64, 100, 33, 10], 0.0, False),
    "prefix and rows without keys": ([100, 90], [30, 20], 4, 1, 64, True, [10, 0], 0.0, False),
    "cap": ([190], [260], 4, 2, 128, True, None, 8.0, False),
    "bias": ([140, 77], [140, 150], 12, 2, 64, True, [0, 40], 0.0, True),
    "cap, bias, not causal": ([100, 31], [60, 90], 7, 7, 128, False, None, 20.0, True),
    "long": ([700], [1500], 2, 1, 128, True, [300], 0.0, False),
    "many documents": ([3, 1, 7, 2] * 40, [3, 5, 7, 1] * 40, 4, 2, 64, True, None, 0.0, False),
    # more tiles than two a CU: no teams, no parts
    "many tiles": ([97, 130, 64] * 15, [97, 130, 70] * 15, 16, 16, 64, True, None, 0.0, False),
    "many tiles of four heads": ([97, 130, 64] * 15, [97, 130, 70] * 15, 16, 4, 128, True, [10] * 45, 0.0, False),
    "many tiles, cap and bias": ([97, 130, 64] * 15, [97, 130, 70] * 15, 16, 4, 128, True, None, 9.0, True),
    # two teams of waves, that have several blocks of keys each
    "two teams": ([400, 150], [1600, 600], 64, 16, 128, True, [0, 500], 0.0, False),
    "two teams, cap and bias": ([400], [1000], 96, 96, 64, True, None, 9.0, True),
    "four teams, small heads": ([300], [1100], 96, 96, 64, True, None, 0.0, False),
    "short documents, more tiles than CUs": ([150, 400], [150, 600], 64, 16, 128, True, [0, 500], 0.0, False),
    # two or more parts of the rows, some of them without a step
    "parts": ([300, 20], [300, 700], 8, 2, 128, True, [0, 500], 0.0, False),
    "parts, small heads": ([520], [520], 6, 2, 64, True, None, 12.0, True),
}


def _run(case, dtype, seed=1, scale=0.0, sharp=1.0, fused=False, grad=True, stream=None):
    rows, keys, H, Hkv, D, causal, prefix, cap, bias = case
    n, m = sum(rows), sum(keys)
    tail = 5  # rows behind the last document
    q, q64 = normal(seed, (n + tail, H, D), dtype, sharp)
    k, k64 = normal(seed + 1, (m + tail, Hkv, D), dtype)
    v, v64 = normal(seed + 2, (m + tail, Hkv, D), dtype)
    do, do64 = normal(seed + 3, (n + tail, H, D), dtype)
    for x in (k, v):  # what no row sees may hold anything
        x[m:] = float("nan")
    slopes = (2.0 ** -np.arange(1, H + 1)).astype(np.float32) if bias else None
    sc = oda.Scores(scale or None, cap, slopes, causal)
    want = doc_reference(q64[:n], k64[:m], v64[:m], rows, keys, sc, prefix or [0] * len(rows), dtype,
                         do64[:n] if grad else None)
    dev = {}
    for name, x in (("q", q), ("k", k), ("v", v)):
        if fused:  # a part of a wider tensor
            wide = torch.full((x.shape[0], x.shape[1] + 2, D), float("nan"), dtype=x.dtype)
            wide[:, 1:-1] = x
            dev[name] = wide.to(DEV)[:, 1:-1]
        else:
            dev[name] = x.to(DEV)
    mark = 17.0
    o = torch.full((n + tail, H, D), mark, dtype=TORCH[dtype], device=DEV)
    lse = torch.full((H, n + tail), mark, device=DEV)
    d = {x: torch.full_like(dev[x].contiguous(), mark) for x in ("q", "k", "v")}
    if fused:
        d = {x: torch.full((t.shape[0], t.shape[1] + 1, D), mark, dtype=t.dtype, device=DEV)[:, 1:] for x, t in d.items()}
    p = {"prefix": None if prefix is None else ints(prefix), "slopes": None if slopes is None else torch.tensor(slopes, device=DEV)}
    a = csg.DocAttn(H, Hkv, D, dtype, causal=causal, scale=scale, softcap=cap)
    qp, kp = ints(pointers(rows)), ints(pointers(keys))
    torch.cuda.synchronize()
    a.forward(dev["q"], dev["k"], dev["v"], qp, kp, o, lse, stream=stream, **p)
    if grad:
        ws = torch.full((a.workspace_bytes(n + tail, m + tail),), 255, dtype=torch.uint8, device=DEV)  # NaN
        torch.cuda.synchronize()
        a.backward(dev["q"], dev["k"], dev["v"], qp, kp, o, lse, do.to(DEV), d["q"], d["k"], d["v"], ws, stream=stream, **p)
    torch.cuda.synchronize()
    got = {"o": (o[:n], o[n:]), "lse": (lse[:, :n], lse[:, n:])}
    if grad:
        got.update(dq=(d["q"][:n], d["q"][n:]), dk=(d["k"][:m], d["k"][m:]), dv=(d["v"][:m], d["v"][m:]))
    for name, (x, behind) in got.items():
        close(x, *want[name], what=name)
        assert bool((behind == mark).all()), "%s: rows behind the last document were written" % name
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", CASES)
def test_documents(name, dtype):
    _run(CASES[name], dtype)


@pytest.mark.parametrize("name", ["edges of 128", "prefix", "cap, bias, not causal"])
def test_parts_of_wider_tensors(name):
    _run(CASES[name], "bf16", fused=True)


def test_given_scale_and_sharp_scores():
    _run(CASES["prefix"], "bf16", scale=0.3, sharp=4.0)
    _run(CASES["prefix"], "f16", scale=0.3, sharp=4.0)


def test_other_stream_and_same_bits():
    st = torch.cuda.Stream(device=DEV)
    one = _run(CASES["prefix"], "bf16", stream=st)
    two = _run(CASES["prefix"], "bf16")
    for name in one:
        assert torch.equal(one[name][0], two[name][0]), name


def test_gradient_against_differences():
    """Directional derivatives of sum(do . o), by central differences of the fp64 definition."""
    case = CASES["prefix"]
    rows, keys, H, Hkv, D, causal, prefix, cap, bias = case
    got = _run(case, "bf16")
    n, m = sum(rows), sum(keys)
    x = {"dq": normal(1, (n + 5, H, D), "bf16")[1][:n], "dk": normal(2, (m + 5, Hkv, D), "bf16")[1][:m],
         "dv": normal(3, (m + 5, Hkv, D), "bf16")[1][:m]}
    do = normal(4, (n + 5, H, D), "bf16")[1][:n]
    want = doc_reference(x["dq"], x["dk"], x["dv"], rows, keys, oda.Scores(), prefix, "bf16", do)
    rng = np.random.default_rng(9)
    for name in x:
        w = rng.standard_normal(x[name].shape)
        f = []
        for h in (1e-4, -1e-4):
            y = {**x, name: x[name] + h * w}
            f.append((doc_reference(y["dq"], y["dk"], y["dv"], rows, keys, oda.Scores(), prefix, "bf16")["o"][0] * do).sum())
        # the gradient's own bounds, and 1e-6 of the terms' size for the differences
        g = f64(got[name][0])
        allowed = (want[name][1] * np.abs(w)).sum() + 1e-6 * np.abs(g * w).sum()
        assert abs((f[0] - f[1]) / 2e-4 - (g * w).sum()) <= allowed, name


@pytest.mark.parametrize("rows", [3, 700])
def test_no_keys_at_all(rows):
    """Rows without a key in the call: output and gradient 0, log-sum-exp -inf; and keys without rows."""
    H, Hkv, D = 32, 8, 128
    a = csg.DocAttn(H, Hkv, D, "bf16")
    for n, m in ((rows, 0), (0, rows)):
        q, k, v, do = (normal(i, s, "bf16")[0].to(DEV)
                       for i, s in enumerate(((n, H, D), (m, Hkv, D), (m, Hkv, D), (n, H, D))))
        o, lse = torch.full_like(q, 17.0), torch.full((H, n), 17.0, device=DEV)
        d = [torch.full_like(t, 17.0) for t in (q, k, v)]
        ws = torch.full((max(16, a.workspace_bytes(n, m)),), 255, dtype=torch.uint8, device=DEV)
        qp, kp = ints([0, n]), ints([0, m])
        a.forward(q, k, v, qp, kp, o, lse)
        a.backward(q, k, v, qp, kp, o, lse, do, *d, ws)
        torch.cuda.synchronize()
        assert all(bool((t == 0).all()) for t in (o, *d)) and bool((lse == float("-inf")).all())


def test_masked_keys_may_be_anything():
    """Keys (not values) that the mask hides hold NaN and infinities, also inside a document."""
    H, D, n = 4, 128, 100
    q, _ = normal(1, (n, H, D), "bf16")
    k, _ = normal(2, (n, 1, D), "bf16")
    v, _ = normal(3, (n, 1, D), "bf16")
    a = csg.DocAttn(H, 1, D, "bf16")
    out = []
    for bad in (0.0, float("nan"), float("inf"), float("-inf")):
        kk = k.clone()
        kk[60:] = bad
        o, lse = torch.zeros((n, H, D), dtype=torch.bfloat16, device=DEV), torch.zeros((H, n), device=DEV)
        a.forward(q.to(DEV), kk.to(DEV), v.to(DEV), ints([0, n]), ints([0, n]), o, lse)
        torch.cuda.synchronize()
        out.append((o[:60].clone(), lse[:, :60].clone()))
    for o, lse in out[1:]:
        assert torch.equal(o, out[0][0]) and torch.equal(lse, out[0][1])


def test_other_documents_may_be_anything():
    H, D = 2, 64
    rows = [40, 50, 30]
    q, _ = normal(1, (120, H, D), "f16")
    k, _ = normal(2, (120, 1, D), "f16")
    v, _ = normal(3, (120, 1, D), "f16")
    do, _ = normal(4, (120, H, D), "f16")
    a = csg.DocAttn(H, 1, D, "f16")
    p = ints(pointers(rows))
    out = []
    for bad in (0.0, float("nan")):
        x = [t.clone() for t in (q, k, v, do)]
        for t in x:
            t[40:90] = bad
        x = [t.to(DEV) for t in x]
        o, lse = torch.zeros_like(x[0]), torch.zeros((H, 120), device=DEV)
        d = [torch.zeros_like(t) for t in x[:3]]
        ws = torch.zeros(a.workspace_bytes(120, 120), dtype=torch.uint8, device=DEV)
        a.forward(x[0], x[1], x[2], p, p, o, lse)
        a.backward(x[0], x[1], x[2], p, p, o, lse, x[3], *d, ws)
        torch.cuda.synchronize()
        out.append([torch.cat([t[:40], t[90:]]) for t in (o, *d)])
    for one, two in zip(*out):
        assert torch.equal(one, two)


def test_far_rows():
    """Rows 16 MiB apart, elements beyond 2^32 of one tensor, bit for bit as dense ones."""
    H, Hkv, D, n, stride = 4, 2, 64, 600, 1 << 23
    x = [normal(i, (n, h, D), "bf16")[0].to(DEV) for i, h in enumerate((H, Hkv, Hkv, H))]
    a = csg.DocAttn(H, Hkv, D, "bf16")
    p = ints([0, 50, n])
    o, lse = torch.zeros((n, H, D), dtype=torch.bfloat16, device=DEV), torch.zeros((H, n), device=DEV)
    ws = torch.zeros(a.workspace_bytes(n, n), dtype=torch.uint8, device=DEV)
    d = [torch.zeros_like(t) for t in x[:3]]
    a.forward(*x[:3], p, p, o, lse)
    a.backward(*x[:3], p, p, o, lse, x[3], *d, ws)
    torch.cuda.synchronize()
    wide = torch.empty((n, stride), dtype=torch.bfloat16, device=DEV)
    far, at = [], 0
    for t in x[:3] + d:
        w = t.shape[1] * D
        far.append(wide[:, at:at + w].unflatten(1, (t.shape[1], D)))
        at += w
    for t, f in zip(x[:3], far):
        f.copy_(t)
    o2, lse2 = torch.zeros_like(o), torch.zeros_like(lse)
    a.forward(*far[:3], p, p, o2, lse2)
    a.backward(*far[:3], p, p, o2, lse2, x[3], *far[3:], ws)
    torch.cuda.synchronize()
    for one, two in zip((o, lse, *d), (o2, lse2, *far[3:])):
        assert torch.equal(one, two)


def test_lowest_scores():
    """Scores of the type's lowest values and of -inf: weights stay a distribution."""
    H, D, n = 1, 64, 70
    q = torch.zeros((n, H, D), dtype=torch.bfloat16)
    k = torch.zeros((n, 1, D), dtype=torch.bfloat16)
    q[..., 0] = 1.0
    k[:, 0, 0] = torch.finfo(torch.bfloat16).min
    k[3, 0, 0] = float("-inf")
    v, v64 = normal(3, (n, 1, D), "bf16")
    o, lse = torch.zeros((n, H, D), dtype=torch.bfloat16, device=DEV), torch.zeros((H, n), device=DEV)
    csg.DocAttn(H, 1, D, "bf16", causal=False, scale=1.0).forward(q.to(DEV), k.to(DEV), v.to(DEV), ints([0, n]), ints([0, n]), o, lse)
    torch.cuda.synchronize()
    # every key but the fourth weighs the same
    want = np.delete(v64[:, 0], 3, axis=0).mean(axis=0)
    size = np.abs(v64).max()
    assert np.abs(f64(o)[:, 0] - want).max() <= 3 * 2.0 ** -8 * size
    assert bool((lse < -3e38).all())


def test_captured_and_replayed():
    """One graph of forward and backward, replayed with other bounds, values and eager work between."""
    H, Hkv, D, n = 4, 2, 64, 200
    a = csg.DocAttn(H, Hkv, D, "bf16")
    x = [torch.zeros((n, h, D), dtype=torch.bfloat16, device=DEV) for h in (H, Hkv, Hkv, H)]
    p = ints([0, 100, 200])
    o, lse = torch.zeros_like(x[0]), torch.zeros((H, n), device=DEV)
    d = [torch.zeros_like(t) for t in x[:3]]
    ws = torch.zeros(a.workspace_bytes(n, n), dtype=torch.uint8, device=DEV)

    def both(stream):
        a.forward(*x[:3], p, p, o, lse, stream=stream)
        a.backward(*x[:3], p, p, o, lse, x[3], *d, ws, stream=stream)

    st = torch.cuda.Stream(device=DEV)
    both(st)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        both(st)
    for seed, bounds in ((1, [0, 100, 200]), (2, [0, 1, 200]), (3, [0, 0, 150])):
        for i, t in enumerate(x):
            t.copy_(normal(10 * seed + i, tuple(t.shape), "bf16")[0])
        p.copy_(ints(bounds))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (o, lse, *d)]
        for t in (o, lse, *d):
            t.zero_()
        torch.cuda.synchronize()
        both(None)
        torch.cuda.synchronize()
        end = bounds[-1]
        for one, two in zip(got, (o, lse, *d)):
            if one.shape[0] == n:
                assert torch.equal(one[:end], two[:end])
            else:
                assert torch.equal(one[:, :end], two[:, :end])


def test_two_streams_at_once():
    """Two calls with their own workspaces on two streams, bit for bit as one after the other."""
    H, Hkv, D, n = 8, 2, 128, 700
    a = csg.DocAttn(H, Hkv, D, "bf16")
    p = ints([0, 300, n])
    sets = []
    for s in (1, 2):
        x = [normal(10 * s + i, (n, h, D), "bf16")[0].to(DEV) for i, h in enumerate((H, Hkv, Hkv, H))]
        sets.append((x, torch.zeros_like(x[0]), torch.zeros((H, n), device=DEV), [torch.zeros_like(t) for t in x[:3]],
                     torch.zeros(a.workspace_bytes(n, n), dtype=torch.uint8, device=DEV)))

    def both(s, stream):
        x, o, lse, d, ws = s
        a.forward(*x[:3], p, p, o, lse, stream=stream)
        a.backward(*x[:3], p, p, o, lse, x[3], *d, ws, stream=stream)

    torch.cuda.synchronize()
    want = []
    for s in sets:
        both(s, None)
        torch.cuda.synchronize()
        want.append([t.clone() for t in (s[1], s[2], *s[3])])
        for t in (s[1], s[2], *s[3]):
            t.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(device=DEV) for _ in sets]
    for _ in range(3):
        for s, st in zip(sets, streams):
            both(s, st)
    torch.cuda.synchronize()
    for s, w in zip(sets, want):
        for one, two in zip((s[1], s[2], *s[3]), w):
            assert torch.equal(one, two)
