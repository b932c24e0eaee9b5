"""The order of the roundings of a key that goes into the 4-bit cache."""
import math

import numpy as np
import pytest

import paper_2601_20595_amd as csg
from oracle import cache4

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    from attn_util import DEV, TORCH, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_keys_roundings(dtype, pairs):
    """A rotated key is rounded to 32 bits, then to the type, then to 4 bits: elements that the second rounding puts on a
    border, and a single rounding to the type beside it."""
    step = {"bf16": 2.0 ** -7, "f16": 2.0 ** -10}[dtype]  # of values in 1 .. 2
    D, rot = 64, 16
    freq, key, codes = np.zeros(8), np.zeros(D), np.zeros(D, dtype=int)
    for i, (border, up) in enumerate([(0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)]):
        ulp = step * 2.0 ** math.floor(math.log2(border))
        # half a step of the type and 2^-26 (of 1 .. 2; half a step of fp32 is 2^-24) more, on the side where the code changes
        x = border + (-1 if up else 1) * 0.5 * ulp * (1 + 2.0 ** -15 * (2.0 ** -3 if dtype == "bf16" else 1))
        direct = border + (-1 if up else 1) * ulp
        assert abs(x - direct) < abs(x - border)  # (a single rounding leaves the border)
        assert float(torch.tensor(x, dtype=torch.float64).float().to(TORCH[dtype])) == border
        at = 2 * i if pairs else i
        key[at] = 6.5
        freq[i] = math.acos(x / 6.5)  # (the pair's other element is 0, and becomes 6.5 sin)
        assert abs(6.5 * math.cos(freq[i]) - x) < 2.0 ** -45
        codes[at] = cache4.quantise(np.array([border, 7.0] + [0.0] * 30), "bf16")[0][0]
        other = cache4.quantise(np.array([direct, 7.0] + [0.0] * 30), "bf16")[0][0]
        assert codes[at] != other
    key[16:32] = 7.0  # sets the scale
    k = torch.tensor(key).to(TORCH[dtype]).view(1, 1, D)
    c = csg.PagedCache4(1, 1, D, dtype, 1, 16, 1, 1)
    kp, vp = (torch.zeros((1, 1, 16 * 34), dtype=torch.uint8, device=DEV) for _ in range(2))
    # position 1: the angle is the frequency
    c.append(kp, vp, k.to(DEV), k.to(DEV), ints([0, 1]), ints([2]), ints([[0]]), inv_freq=torch.tensor(freq, device=DEV), interleaved=pairs)
    torch.cuda.synchronize()
    got, scales = cache4.unpack(kp.cpu().numpy(), 16, D)
    assert scales[0, 0, 1, 0] == 127
    at = [2 * i if pairs else i for i in range(7)]
    assert got[0, 0, 1, at].tolist() == codes[at].tolist()
