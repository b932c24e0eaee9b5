"""Attention over documents and over a paged cache, on the host: refusals (nothing is queued: the
addresses are never read), workspaces, the oracle's own pins, and the kernels' assembly."""
import os
import re

import numpy as np
import pytest

import oracle
import paper_2601_20595_amd as csg
from oracle import doc_attention as oda
from test_kernel_asm import device_asm, divergent_barrier_loops, wide_stores_with_offset_register

P = 1 << 20  # an address that no call reads
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _docs(**change):
    c = csg.csg_doc_attn_cfg(n_heads=8, n_kv_heads=2, head_dim=128, dtype=csg.CSG_BF16, causal=1, n_docs=2, q_rows=100, k_rows=100)
    for k, v in change.items():
        setattr(c, k, v)
    return c


def _cache(**change):
    c = csg.csg_cache_cfg(n_heads=8, n_kv_heads=2, head_dim=128, dtype=csg.CSG_BF16, n_pages=10, page_size=16, batch=2,
                          max_pages=4, tokens=2)
    for k, v in change.items():
        setattr(c, k, v)
    return c


def _status(f, *args, **kw):
    with pytest.raises(csg.CsgError) as e:
        f(*args, **kw)
    return e.value.status


INVALID, UNSUPPORTED = csg.CSG_ERR_INVALID, csg.CSG_ERR_UNSUPPORTED

HEADS = [({"n_heads": 0}, INVALID), ({"n_heads": 7}, INVALID), ({"n_kv_heads": 0}, INVALID), ({"n_kv_heads": -2}, INVALID),
         ({"n_heads": 1 << 20}, INVALID), ({"dtype": 9}, INVALID), ({"dtype": csg.CSG_F32}, UNSUPPORTED),
         ({"head_dim": 96}, UNSUPPORTED), ({"head_dim": 0}, UNSUPPORTED), ({"scale": -1.0}, INVALID),
         ({"scale": float("nan")}, INVALID), ({"scale": float("inf")}, INVALID), ({"softcap": -1.0}, INVALID),
         ({"softcap": float("nan")}, INVALID), ({"softcap": float("inf")}, INVALID),
         ({"scale": 1e-40}, INVALID), ({"scale": 3e38}, INVALID), ({"softcap": 1e-40}, INVALID), ({"softcap": 3e38}, INVALID),
         ({"scale": 1e30, "softcap": 1e-10}, INVALID), ({"scale": 1e-30, "softcap": 1e10}, INVALID)]
DOCS = HEADS + [({"causal": 2}, INVALID), ({"n_docs": -1}, INVALID), ({"q_rows": -1}, INVALID), ({"k_rows": 1 << 31}, INVALID),
                ({"q_stride": 8 * 128 - 8}, INVALID), ({"k_stride": 2 * 128 + 4}, INVALID), ({"v_stride": (1 << 23) + 8}, UNSUPPORTED),
                ({"n_docs": 1 << 29, "n_heads": 64}, UNSUPPORTED)]


@pytest.mark.parametrize("change, status", DOCS)
def test_documents_refuse(change, status):
    c = _docs(**change)
    assert _status(csg.csg_doc_attn, c, P, P, P, P, P, 0, 0, P, P) == status
    assert _status(csg.csg_doc_attn_grad, c, P, P, P, P, P, 0, 0, P, P, P, P, P, P, P, 1 << 40) == status
    assert _status(csg.csg_doc_attn_grad_workspace, c, -1) == status


@pytest.mark.parametrize("change, status", [({"dq_stride": 8}, INVALID), ({"dk_stride": 2 * 128 + 1}, INVALID),
                                            ({"dv_stride": 1 << 24}, UNSUPPORTED)])
def test_gradients_refuse(change, status):
    assert _status(csg.csg_doc_attn_grad, _docs(**change), P, P, P, P, P, 0, 0, P, P, P, P, P, P, P, 1 << 40) == status


def test_documents_refuse_buffers():
    need = csg.csg_doc_attn_grad_workspace(_docs(), -1)
    assert need >= 2 * 8 * 100 * 4
    for i in (0, 1, 2, 3, 4, 7, 8):
        args = [P, P, P, P, P, 0, 0, P, P]
        args[i] = 0
        assert _status(csg.csg_doc_attn, _docs(), *args) == INVALID
    for i in (0, 1, 2, 7, 8):
        args = [P, P, P, P, P, 0, 0, P, P]
        args[i] = P + 8
        assert _status(csg.csg_doc_attn, _docs(), *args) == INVALID
    for i in (0, 1, 2, 3, 4, 7, 8, 9, 10, 11, 12, 13):
        args = [P, P, P, P, P, 0, 0, P, P, P, P, P, P, P]
        args[i] = 0
        assert _status(csg.csg_doc_attn_grad, _docs(), *args, need) == INVALID
        args[i] = P + 4
        if i not in (3, 4):
            assert _status(csg.csg_doc_attn_grad, _docs(), *args, need) == INVALID
    assert _status(csg.csg_doc_attn, _docs(), P, P, P, P, P, 0, 0, P, P, device=64) == INVALID
    # nothing to do: no buffer is needed, and no device
    csg.csg_doc_attn(_docs(q_rows=0), 0, 0, 0, 0, 0, 0, 0, 0, 0)
    csg.csg_doc_attn(_docs(n_docs=0), 0, 0, 0, 0, 0, 0, 0, 0, 0)
    csg.csg_doc_attn_grad(_docs(q_rows=0, k_rows=0), 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)


CACHE = HEADS[:8] + [({"n_pages": 0}, INVALID), ({"page_size": 0}, INVALID), ({"page_size": 8}, UNSUPPORTED),
                     ({"page_size": 48}, UNSUPPORTED), ({"batch": -1}, INVALID), ({"max_pages": 0}, INVALID),
                     ({"tokens": -1}, INVALID), ({"tokens": 1 << 31}, INVALID), ({"tokens": 1 << 24}, UNSUPPORTED), ({"n_groups": -1}, INVALID),
                     ({"max_pages": 1 << 27}, UNSUPPORTED), ({"q_stride": 100}, INVALID)]


@pytest.mark.parametrize("change, status", CACHE)
def test_cache_refuses(change, status):
    c = _cache(**change)
    assert _status(csg.csg_cache_append, c, P, P, P, P, 0, 0, P, P, P, 0) == status
    assert _status(csg.csg_cache_attn, c, P, P, P, P, P, P, 0, 0, 0, P, P, P, 1 << 40) == status
    assert _status(csg.csg_cache_attn_workspace, c, -1) == status


def test_append_refuses():
    good = [P, P, P, P, P, P, P, P, P, P]
    for change in ({"rot_dim": 144}, {"rot_dim": 8}, {"rot_dim": -16}, {"interleaved": 2}, {"k_stride": 8}, {"v_stride": 2 * 128 + 4}):
        assert _status(csg.csg_cache_append, _cache(**change), *good) == INVALID
    for i in (0, 1, 2, 3, 6, 7, 8):
        args = list(good)
        args[i] = 0
        assert _status(csg.csg_cache_append, _cache(), *args) == INVALID
    for i in (0, 1, 2, 3, 4, 5):
        args = list(good)
        args[i] = P + 2
        assert _status(csg.csg_cache_append, _cache(), *args) == INVALID
    args = list(good)
    args[9] = 0
    assert _status(csg.csg_cache_append, _cache(rot_dim=64), *args) == INVALID       # no frequencies
    args = list(good)
    args[5] = 0
    assert _status(csg.csg_cache_append, _cache(), *args) == INVALID                 # q without q_out
    assert _status(csg.csg_cache_append, _cache(q_stride=8 * 128 + 8), *good) == INVALID  # q_out is q, which is not dense
    csg.csg_cache_append(_cache(tokens=0), *([0] * 10))


def test_cache_attention_refuses():
    need = csg.csg_cache_attn_workspace(_cache(), -1)
    for change, status in HEADS[8:] + [({"n_groups": 3}, INVALID), ({"batch": 2049}, UNSUPPORTED),
                                       ({"batch": 2000, "n_groups": 100}, UNSUPPORTED), ({"tokens": 1 << 29}, UNSUPPORTED)]:
        assert _status(csg.csg_cache_attn, _cache(**change), P, P, P, P, P, P, P, P, 0, P, P, P, 1 << 50) == status
    for i in (0, 1, 2, 3, 4, 5, 9, 11):
        args = [P, P, P, P, P, P, 0, 0, 0, P, P, P]
        args[i] = 0
        assert _status(csg.csg_cache_attn, _cache(), *args, need) == INVALID
    for i in (6, 7):
        args = [P, P, P, P, P, P, P, P, 0, P, P, P]
        args[i] = 0
        assert _status(csg.csg_cache_attn, _cache(n_groups=1), *args, 1 << 40) == INVALID
    csg.csg_cache_attn(_cache(tokens=0), *([0] * 12), 0)
    # more work needs no less
    sizes = [csg.csg_cache_attn_workspace(_cache(tokens=t), -1) for t in (0, 1, 2, 64, 1000)]
    assert sizes == sorted(sizes) and sizes[0] > 0


def test_python_checks():
    torch = pytest.importorskip("torch")
    with pytest.raises(csg.CsgError):
        csg.DocAttn(8, 3, 128, "bf16")
    with pytest.raises(csg.CsgError):
        csg.PagedCache(8, 2, 128, "f32", 4, 16, 1, 1)
    a = csg.DocAttn(8, 2, 128, "bf16")
    x = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # not on a GPU
        a.forward(x, x[:, :2], x[:, :2], torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), x, x)
    with pytest.raises(ValueError):
        a.forward(x[:, :4], x[:, :2], x[:, :2], None, None, x, x)
    with pytest.raises(ValueError):
        a.forward(x.float(), x[:, :2], x[:, :2], None, None, x, x)
    with pytest.raises(ValueError):
        a.forward(x.transpose(0, 2), x[:, :2], x[:, :2], None, None, x, x)


def test_python_checks_elements_and_rows():
    torch = pytest.importorskip("torch")
    x = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    a = csg.DocAttn(8, 8, 128, "bf16")
    with pytest.raises(ValueError, match="rows apart"):  # one row for all
        a.forward(x[:1].expand(4, 8, 128), x, x, None, None, x, x)
    with pytest.raises(ValueError, match="4-byte"):
        csg._arg(torch.zeros(3, dtype=torch.int64), 12, 4, "q_ptr", 0)
    with pytest.raises(ValueError, match="contiguous"):
        csg._arg(torch.zeros((4, 4), dtype=torch.int32)[:, :2], 16, 4, "page_table", 0)
    with pytest.raises(ValueError, match="holds"):
        csg._arg(torch.zeros(3, dtype=torch.int32), 16, 4, "lens", 0)
    with pytest.raises(ValueError, match="GPU"):
        csg._arg(torch.zeros(3, dtype=torch.int32), 12, 4, "lens", 0)
    c = csg.PagedCache(8, 8, 128, "bf16", 4, 16, 2, 5)
    with pytest.raises(ValueError, match="5 pages a row"):
        c._table(torch.zeros((2, 4), dtype=torch.int32))


# ---- the oracle -----------------------------------------------------------------------------
def test_oracle_without_masks_is_the_ring_attention_oracle():
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal(s) for s in ((9, 6, 16), (14, 2, 16), (14, 2, 16)))
    o, lse = oracle.attention(q, k, v)
    got = oda.attention(q, k, v, oda.Scores(causal=False))
    assert np.allclose(got[0], o, rtol=1e-12, atol=1e-13) and np.allclose(got[1], lse, rtol=1e-12)


def test_oracle_masks_by_hand():
    assert oda.visible(2, 4, True).tolist() == [[True, True, True, False], [True] * 4]
    assert oda.visible(3, 2, True).tolist() == [[False, False], [True, False], [True, True]]
    assert oda.visible(3, 3, True, 2).tolist() == [[True, True, False], [True, True, False], [True] * 3]
    assert oda.visible(2, 3, False).all()
    # one visible key: its value, and its score
    q, k, v = np.full((2, 1, 4), 1.0), np.array([[[1.0, 2, 3, 4]], [[9.0, 9, 9, 9]]]), np.array([[[5.0, 6, 7, 8]], [[1.0, 1, 1, 1]]])
    o, lse, _, _ = oda.attention(q, k, v, oda.Scores(0.5, 2.0, np.array([3.0]), True))
    assert np.allclose(o[0, 0], [5, 6, 7, 8]) and np.isclose(lse[0, 0], 2 * np.tanh(5.0 / 2))
    # the other row: its own key without bias, the first at distance 1
    s = np.array([2 * np.tanh(2.5) - 3, 2 * np.tanh(9.0)])
    p = np.exp(s) / np.exp(s).sum()
    assert np.allclose(o[1, 0], p[0] * v[0, 0] + p[1] * v[1, 0])


def test_oracle_gradient_against_differences():
    rng = np.random.default_rng(4)
    sc = oda.Scores(0.4, 3.0, np.array([0.5, 0.25]), True)
    x = [rng.standard_normal(s) for s in ((5, 2, 8), (7, 1, 8), (7, 1, 8))]
    do = rng.standard_normal((5, 2, 8))
    d, _ = oda.attention_grad(*x, do, sc, 2)
    for n in range(3):
        for at in [(0, 0, 0), (4, 0, 3), (2, 0, 7)]:
            f = []
            for h in (1e-5, -1e-5):
                y = [t.copy() for t in x]
                y[n][at] += h
                f.append((oda.attention(*y, sc, 2)[0] * do).sum())
            assert abs((f[0] - f[1]) / 2e-5 - d[n][at]) <= 1e-7 * (1 + np.abs(d[n]).max())


def test_oracle_rotation_keeps_products_of_equal_distance():
    rng = np.random.default_rng(4)
    x, y = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))
    f = 100.0 ** (-np.arange(0, 16, 2) / 16)
    for pairs in (False, True):
        got = [(oda.rotate(x, [p + 3], f, pairs) * oda.rotate(y, [p], f, pairs)).sum() for p in (0, 5, 1000)]
        assert np.allclose(got, got[0])


# ---- the compiled kernels -----------------------------------------------------------------------
@pytest.mark.parametrize("source", ["doc_attn.hip", "cache_attn.hip"])
def test_kernels_barrier_loops_and_stores(source):
    asm = device_asm(os.path.join(ROOT, "paper_2601_20595_amd", "csrc", source))
    assert re.findall(r"^(_Z\S+):", asm, re.M)
    assert divergent_barrier_loops(asm) == []
    assert wide_stores_with_offset_register(asm) == []
