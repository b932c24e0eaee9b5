"""The most keys that attention over each paged cache takes, on the host (addresses are never read)."""
import pytest

import paper_2601_20595_amd as csg
from test_attn_ops_host import P, UNSUPPORTED, _cache, _status

CALLS = {16: (csg.csg_cache_attn_workspace, csg.csg_cache_attn), 4: (csg.csg_cache4_attn_workspace, csg.csg_cache4_attn)}
COST = {16: 4, 4: 10}  # units that beginning a task costs, beside its blocks of 32 keys


def _most_pages(bits, batch):
    """Pages of 32 of each of batch sequences whose units still count in 32 bits."""
    tasks = batch // 4 + batch  # (every sequence has a tile, four of which are a task)
    return (2 ** 31 - 1) // tasks - COST[bits] - 1


@pytest.mark.parametrize("bits", CALLS)
@pytest.mark.parametrize("batch", [52, 400, 2000])
def test_as_many_pages_as_the_caches_own_units_allow(bits, batch):
    workspace, attn = CALLS[bits]
    most = _most_pages(bits, batch)
    c = _cache(batch=batch, tokens=0, max_pages=most, page_size=32)
    assert workspace(c, -1) > 0
    attn(c, *([0] * 12), 0)  # (nothing to do: no buffer is needed)
    c.max_pages = most + 1
    assert _status(workspace, c, -1) == UNSUPPORTED
    assert _status(attn, c, P, P, P, P, P, P, 0, 0, 0, P, P, P, 1 << 40) == UNSUPPORTED


def test_each_class_checks_its_own_limit():
    shape = (8, 2, 128, "bf16", 10, 32, 52)
    for kind, bits in ((csg.PagedCache, 16), (csg.PagedCache4, 4)):
        kind(*shape, _most_pages(bits, 52))
        with pytest.raises(csg.CsgError):
            kind(*shape, _most_pages(bits, 52) + 1)
