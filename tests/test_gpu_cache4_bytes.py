"""What append writes into the 4-bit cache, byte for byte: scales, codes, their places, and nothing beside them."""
import numpy as np
import pytest

import paper_2601_20595_amd as csg
from oracle import cache4

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from attn_util import DEV, TORCH, ints, normal

pytestmark = pytest.mark.gpu
INFINITY = {"bf16": 0x7F80, "f16": 0x7C00}
FILL = 0x5A


def _rows(dtype, D):
    """[rows, 2, D] of the type: all patterns in order and mixed, zeros of both signs, values that several scales hold,
    sizes next to where the scale changes, single elements of every size."""
    rng = np.random.default_rng(D)
    every = np.arange(65536, dtype=np.uint16)
    finite = every[(every & 0x7FFF) < INFINITY[dtype]]

    def bits(x):
        return torch.as_tensor(np.asarray(x, dtype=np.float64)).to(TORCH[dtype]).view(torch.int16).numpy().view(np.uint16).reshape(-1)

    lone = np.zeros((len(finite) // 16, 32), dtype=np.uint16)
    lone[np.arange(len(lone)), rng.integers(0, 32, len(lone))] = finite[::16][:len(lone)]
    grid = rng.choice([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], (64, 32)) * rng.choice([1.0, -1.0], (64, 32)) * rng.choice([0.25, 1.0, 8.0], (64, 1))
    few = rng.choice([0.0, 1.0, -2.0], (32, 32))
    top = np.array([6.0, 6.5, 6.96875, 7.0, 7.03125, 7.5, 8.0])[:, None] * rng.choice([-1.0, 1.0], (7, 32)) * rng.choice([1.0, 0.1], (7, 32))
    parts = [finite, rng.permutation(finite), every, np.zeros(64, dtype=np.uint16), np.full(64, 0x8000, dtype=np.uint16), lone.reshape(-1),
             bits(grid), bits(few), bits(top)]
    x = np.concatenate(parts)
    x = np.concatenate([x, np.zeros(-len(x) % (2 * D), dtype=np.uint16)])
    return torch.tensor(x.reshape(-1, 2, D).view(np.int16)).view(TORCH[dtype])


@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_bytes(dtype, D, page):
    v = _rows(dtype, D)
    k = v.flip(0).contiguous()
    n, row = len(v), D // 2 + D // 32
    start = 5  # (the first rows and the last are nobody's new tokens)
    width = -(-(n + start) // page)
    order = np.random.default_rng(1).permutation(width + 1)[:width]
    c = csg.PagedCache4(2, 2, D, dtype, width + 1, page, 1, width)
    kp, vp = (torch.full((width + 1, 2, page * row), FILL, dtype=torch.uint8, device=DEV) for _ in range(2))
    c.append(kp, vp, k.to(DEV), v.to(DEV), ints([0, n]), ints([n + start]), ints([order.tolist()]))
    torch.cuda.synchronize()
    at = np.arange(start, n + start)
    for got, x in ((kp, k), (vp, v)):
        want_codes, want_scales = cache4.unpack(np.full((width + 1, 2, page * row), FILL, dtype=np.uint8), page, D)
        want_codes, want_scales = want_codes.copy(), want_scales.copy()
        want_codes[order[at // page], :, at % page], want_scales[order[at // page], :, at % page] = cache4.quantise(x.double().numpy(), dtype)
        codes, scales = cache4.unpack(got.cpu().numpy(), page, D)
        assert np.array_equal(scales, want_scales)
        # a zero may have either sign; codes under a NaN's scale stand for nothing
        free = (((codes | want_codes) & 7) == 0) | (np.repeat(scales, 32, axis=-1) == cache4.NAN)
        assert np.array_equal(codes[~free], want_codes[~free])


def test_scales_of_neighbouring_rows():
    """They share words, and rows of one page may be written at once: all of them arrive."""
    D, page, H = 64, 16, 3
    n = 40
    x, x64 = normal(1, (2 * n, H, D), "bf16")
    c = csg.PagedCache4(H, H, D, "bf16", 6, page, 2, 3)
    kp, vp = (torch.full((6, H, page * 34), FILL, dtype=torch.uint8, device=DEV) for _ in range(2))
    table = np.array([[4, 0, 2], [1, 5, 3]])
    c.append(kp, vp, x.to(DEV), x.to(DEV), ints([0, n, 2 * n]), ints([n, n]), ints(table.tolist()))
    torch.cuda.synchronize()
    codes, scales = cache4.quantise(x64, "bf16")
    for got in (kp, vp):
        gc, gs = cache4.unpack(got.cpu().numpy(), page, D)
        for b in range(2):
            i = np.arange(n)
            assert np.array_equal(gs[table[b][i // page], :, i % page], scales[n * b:n * b + n])
            same = (gc[table[b][i // page], :, i % page] == codes[n * b:n * b + n]) | (codes[n * b:n * b + n] & 7 == 0)
            assert same.all()
