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
