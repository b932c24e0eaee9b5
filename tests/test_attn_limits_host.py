"""Sizes that attention over documents and over a cache takes, on the host (addresses are never read)."""
import pytest

import paper_2601_20595_amd as csg


def _cache(**change):
    c = csg.csg_cache_cfg(n_heads=64, n_kv_heads=8, head_dim=128, dtype=csg.CSG_BF16, n_pages=10, page_size=64, batch=2,
                          max_pages=4096, tokens=2)
    for k, v in change.items():
        setattr(c, k, v)
    return c


def test_a_cache_takes_a_prompt_of_half_a_million_tokens():
    assert csg.csg_cache_attn_workspace(_cache(tokens=1 << 17), -1) > 0
    assert csg.csg_cache_attn_workspace(_cache(tokens=1 << 19, max_pages=1 << 13), -1) > 0
    with pytest.raises(csg.CsgError) as e:
        csg.csg_cache_attn_workspace(_cache(tokens=(1 << 19) + 1), -1)
    assert e.value.status == csg.CSG_ERR_UNSUPPORTED


@pytest.mark.parametrize("heads, kv, d", [(32, 8, 128), (12, 12, 64), (64, 8, 64), (5, 1, 128), (16, 16, 128)])
def test_a_gradients_workspace_serves_fewer_rows_too(heads, kv, d):
    """Fewer keys may be cut into more parts: more rows or keys never need less."""
    def need(q, k):
        c = csg.csg_doc_attn_cfg(n_heads=heads, n_kv_heads=kv, head_dim=d, dtype=csg.CSG_BF16, causal=1, n_docs=1, q_rows=q, k_rows=k)
        return csg.csg_doc_attn_grad_workspace(c, -1)

    sizes = [0, 1, 100, 128, 129, 500, 700, 1024, 1500, 2047, 2049, 3000, 4096, 4097, 5000, 6000, 8191, 8192, 20000, 70000]
    table = [[need(q, k) for k in sizes] for q in sizes]
    for row in table:
        assert row == sorted(row)
    for column in zip(*table):
        assert list(column) == sorted(column)


def test_joined_is_a_truth_value():
    c = csg.csg_doc_attn_cfg(n_heads=8, n_kv_heads=2, head_dim=128, dtype=csg.CSG_BF16, n_docs=1, q_rows=1, k_rows=1, joined=2)
    with pytest.raises(csg.CsgError) as e:
        csg.csg_doc_attn_grad(c, *([1 << 20] * 5), 0, 0, *([1 << 20] * 7), 1 << 30)
    assert e.value.status == csg.CSG_ERR_INVALID and "joined" in str(e.value)
