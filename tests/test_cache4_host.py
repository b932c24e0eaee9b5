"""The cache in 4 bits on the host: the oracle's own pins, refusals (nothing is queued: the addresses
are never read) and the kernels' assembly."""
import os

import numpy as np
import pytest

import paper_2601_20595_amd as csg
from oracle import cache4
from test_attn_ops_host import CACHE, INVALID, P, UNSUPPORTED, _cache, _status
from test_kernel_asm import device_asm, divergent_barrier_loops, wide_stores_with_offset_register

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _block(*x):
    return np.array(list(x) + [0.0] * (32 - len(x)))


def test_oracle_by_hand():
    # 7 = 7 * 2^0: scale 1; ties 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5 go to the even code
    codes, scale = cache4.quantise(_block(7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.26, -6.9), "bf16")
    assert scale[0] == 127 and codes[:10].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 9, 15]
    # just beyond 7: twice the scale
    codes, scale = cache4.quantise(_block(7.03125, 1.0), "bf16")
    assert scale[0] == 128 and codes[:2].tolist() == [6, 1]
    assert cache4.values(codes, scale)[:3].tolist() == [8.0, 1.0, 0.0]
    assert cache4.quantise(_block(), "bf16")[1][0] == 2 and cache4.quantise(_block(), "f16")[1][0] == 104
    # the ends of the ranges: saturation, and values that vanish
    assert cache4.values(*cache4.quantise(_block(3.3e38), "bf16"))[0] == 6.0 * 2.0 ** 125
    assert cache4.values(*cache4.quantise(_block(65504.0), "f16"))[0] == 49152.0
    assert cache4.values(*cache4.quantise(_block(2.0 ** -24), "f16"))[0] == 2.0 ** -24
    for bad in (np.nan, np.inf, -np.inf):
        codes, scale = cache4.quantise(_block(bad, 1.0), "f16")
        assert scale[0] == 255 and np.isnan(cache4.values(codes, scale)).all()


def test_oracle_is_nearest():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 64)) * 10.0 ** rng.uniform(-3, 3, (200, 1))
    codes, scale = cache4.quantise(x, "bf16")
    got = cache4.values(codes, scale)
    unit = np.repeat(2.0 ** (scale.astype(float) - 127), 32, axis=-1)
    # no value of the block's grid is nearer, and half the scale would leave an element beyond 7 times it
    every = unit[..., None] * np.concatenate([cache4.GRID, -cache4.GRID])
    assert (np.abs(got - x) <= np.abs(every - x[..., None]).min(axis=-1)).all()
    top = np.abs(x).reshape(200, 2, 32).max(axis=-1)
    assert (top <= 7 * unit[:, ::32]).all() and (top > 3.5 * unit[:, ::32]).all()
    pages = cache4.pack(codes.reshape(25, 1, 8, 64), scale.reshape(25, 1, 8, 2))
    back = cache4.unpack(pages, 8, 64)
    assert np.array_equal(back[0].reshape(200, 64), codes) and np.array_equal(back[1].reshape(200, 2), scale)


@pytest.mark.parametrize("change, status", CACHE)
def test_refuses(change, status):
    c = _cache(**change)
    assert _status(csg.csg_cache4_append, c, P, P, P, P, 0, 0, P, P, P, 0) == status
    assert _status(csg.csg_cache4_attn, c, P, P, P, P, P, P, 0, 0, 0, P, P, P, 1 << 40) == status
    assert _status(csg.csg_cache4_attn_workspace, c, -1) == status
    if "q_stride" not in change and change != {"tokens": 1 << 24}:
        assert _status(csg.csg_cache4_read, c, P, P, P, P, P, P, P) == status


def test_refuses_buffers_and_options():
    for change in ({"rot_dim": 144}, {"rot_dim": 8}, {"interleaved": 2}, {"k_stride": 8}, {"v_stride": 2 * 128 + 4}):
        assert _status(csg.csg_cache4_append, _cache(**change), *[P] * 10) == INVALID
    for change in ({"k_stride": 8}, {"v_stride": 2 * 128 + 4}):
        assert _status(csg.csg_cache4_read, _cache(**change), *[P] * 7) == INVALID
    assert _status(csg.csg_cache4_read, _cache(k_stride=(1 << 23) + 8), *[P] * 7) == UNSUPPORTED
    assert _status(csg.csg_cache4_read, _cache(n_heads=65536, n_kv_heads=65536, tokens=1 << 26), *[P] * 7) == UNSUPPORTED
    for i in range(7):
        assert _status(csg.csg_cache4_read, _cache(), *[0 if j == i else P for j in range(7)]) == INVALID
        if i not in (2, 3, 4):
            assert _status(csg.csg_cache4_read, _cache(), *[P + 8 if j == i else P for j in range(7)]) == INVALID
    for i in (0, 1, 2, 3, 6, 7, 8):
        assert _status(csg.csg_cache4_append, _cache(), *[0 if j == i else P for j in range(10)]) == INVALID
    for i in (0, 1, 2, 3, 4, 5, 9, 11):
        args = [P, P, P, P, P, P, 0, 0, 0, P, P, P]
        args[i] = 0
        assert _status(csg.csg_cache4_attn, _cache(), *args, 1 << 40) == INVALID
    # nothing to do: no buffer is needed, and no device
    csg.csg_cache4_append(_cache(tokens=0), *([0] * 10))
    csg.csg_cache4_read(_cache(tokens=0), *([0] * 7))
    csg.csg_cache4_attn(_cache(tokens=0), *([0] * 12), 0)


def test_python_refuses():
    torch = pytest.importorskip("torch")
    c = csg.PagedCache4(4, 2, 64, "bf16", 8, 16, 2, 3)
    ptr, lens, table = (torch.zeros(s, dtype=torch.int32) for s in ((3,), (2,), (2, 3)))
    k = torch.zeros((5, 2, 64), dtype=torch.bfloat16)
    pages = torch.zeros((8, 2, 16 * 34), dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        c.read(pages, pages, ptr, lens, table, k, k)
    with pytest.raises(ValueError, match=r"\(5, 2, 64\)|rows"):
        c.read(pages, pages, ptr, lens, table, k[:, :1], k)
    for bad in (pages[:7], pages.to(torch.float16)):
        with pytest.raises(ValueError):
            csg._arg(bad, *c._pages, "k_pages", 0)
    with pytest.raises(csg.CsgError):
        csg.PagedCache4(4, 2, 96, "bf16", 8, 16, 2, 3)


def test_kernels_assembly():
    asm = device_asm(os.path.join(ROOT, "paper_2601_20595_amd", "csrc", "cache4.hip"))
    assert divergent_barrier_loops(asm) == []
    assert wide_stores_with_offset_register(asm) == []
    assert "scratch_" not in asm, "a kernel spills"
