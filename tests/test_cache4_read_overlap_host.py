"""Outputs of the 4-bit cache's read that share memory with each other or with the pages are refused, on the host (addresses are
never read; a call that is not refused for that ends at the device, which there is not)."""
import pytest

import paper_2601_20595_amd as csg
from test_attn_ops_host import P, _cache, _status

ROW = 2 * 2 * 128  # bytes of a row of both heads
KP, VP = P, P + (1 << 20)
K = P + (1 << 24)


def _overlaps(k, v, kp=KP, vp=VP, **change):
    c = _cache(tokens=change.pop("tokens", 5), **change)
    with pytest.raises(csg.CsgError) as e:
        csg.csg_cache4_read(c, kp, vp, P, P, P, k, v, device=64)
    assert e.value.status == csg.CSG_ERR_INVALID
    assert ("overlap" in str(e.value)) != ("device 64" in str(e.value))
    return "overlap" in str(e.value)


@pytest.mark.parametrize("off, meets", [(0, True), (16, True), (ROW - 16, True), (ROW, True), (5 * ROW - 16, True), (5 * ROW, False),
                                        (5 * ROW + 16, False)])
def test_dense_rows(off, meets):
    assert _overlaps(K, K + off) == meets and _overlaps(K + off, K) == meets


@pytest.mark.parametrize("tokens", [1, 2, 5])
def test_parts_of_a_wider_tensor(tokens):
    wide = 5 * ROW  # bytes from row to row
    kw = {"tokens": tokens, "k_stride": wide // 2, "v_stride": wide // 2}
    for off in range(0, (tokens + 1) * wide, 16):
        # beside each other: at least a row apart, and a row of the other's end
        part = off % wide
        meets = off < (tokens - 1) * wide + ROW and (part < ROW or (part > wide - ROW and off < (tokens - 1) * wide))
        assert _overlaps(K, K + off, **kw) == meets and _overlaps(K + off, K, **kw) == meets, off


def test_rows_of_different_strides():
    kw = {"k_stride": ROW // 2, "v_stride": 3 * ROW // 2}
    assert _overlaps(K, K, **kw) and _overlaps(K, K + 4 * ROW, **kw) and not _overlaps(K, K + 5 * ROW, **kw)
    assert _overlaps(K + 12 * ROW, K, **kw) and not _overlaps(K + 13 * ROW, K, **kw)
    assert not _overlaps(K + ROW, K, tokens=1, **kw) and _overlaps(K + ROW - 16, K, tokens=1, **kw)


@pytest.mark.parametrize("dtype, D", [(csg.CSG_BF16, 128), (csg.CSG_F16, 64)])
def test_pages(dtype, D):
    pages, row, far = 10 * 2 * 16 * (D // 2 + D // 32), 4 * D, K + (1 << 20)
    kw = {"dtype": dtype, "head_dim": D, "k_stride": 10 * D, "v_stride": 10 * D}
    for at in (KP, VP):
        for place in (lambda x: (x, far), lambda x: (far, x)):
            assert _overlaps(*place(at), **kw) and _overlaps(*place(at + pages - 16), **kw) and not _overlaps(*place(at + pages), **kw)
            last = 4 * 20 * D  # the last row's first byte
            assert _overlaps(*place(at - last - row + 16), **kw) and not _overlaps(*place(at - last - row), **kw)


def test_other_refusals_come_first():
    assert _status(csg.csg_cache4_read, _cache(k_stride=8), *[P] * 7) == csg.CSG_ERR_INVALID
    assert _status(csg.csg_cache4_read, _cache(k_stride=(1 << 23) + 8), *[P] * 7) == csg.CSG_ERR_UNSUPPORTED
    csg.csg_cache4_read(_cache(tokens=0), *[P] * 7)  # (nothing to do)
