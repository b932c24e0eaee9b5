"""Helpers for the tests of attention over documents and over a paged cache."""
from __future__ import annotations

import numpy as np
import torch

from oracle import doc_attention as oda

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16}
# half a step relative to the value; a weight below the smallest normal number (f16: 2^-14) is
# rounded to a multiple of 2^-24, half of which is the most it is off (bf16: nothing to speak of)
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"bf16": 0.0, "f16": 2.0 ** -25}


def normal(seed, shape, dtype, scale=1.0):
    """Values of the type, made on the CPU: (tensor, the same in fp64)."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(shape, generator=g) * scale).to(TORCH[dtype])
    return x, x.double().numpy()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def pointers(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(int)


def f64(t):
    return t.detach().cpu().double().numpy()


def close(got, want, bound, what):
    """Elementwise |got - want| <= bound; -inf only where -inf is wanted."""
    got = f64(got) if torch.is_tensor(got) else got
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), "%s: other places are not finite" % what
    assert np.array_equal(got[~fine], want[~fine]), what
    off = np.abs(got[fine] - want[fine]) - bound[fine]
    if off.size and off.max() > 0:
        at = np.unravel_index(np.argmax(np.where(fine, np.abs(np.where(fine, got, 0) - np.where(fine, want, 0)) - bound, -1)), want.shape)
        raise AssertionError("%s: off by %.3g at %s, %.3g allowed (%g, wanted %g)"
                             % (what, abs(got[at] - want[at]), at, bound[at], got[at], want[at]))


def doc_reference(q, k, v, rows, keys, sc, prefix, dtype, do=None):
    """Packed documents through the oracle: o, lse and bounds; with do the gradients too."""
    u, tiny = HALF_STEP[dtype], TINY[dtype]
    qp, kp = pointers(rows), pointers(keys)
    out = []
    for t in range(len(rows)):
        r, c = slice(qp[t], qp[t + 1]), slice(kp[t], kp[t + 1])
        x = list(oda.attention(q[r], k[c], v[c], sc, prefix[t], u, tiny))
        if do is not None:
            d, e = oda.attention_grad(q[r], k[c], v[c], do[r], sc, prefix[t], u, tiny)
            x += list(d) + list(e)
        out.append(x)

    def cat(i, axis=0):
        return np.concatenate([x[i] for x in out], axis=axis)

    got = {"o": (cat(0), cat(2)), "lse": (cat(1, 1), cat(3, 1))}
    if do is not None:
        for n, name in enumerate(("dq", "dk", "dv")):
            got[name] = (cat(4 + n), cat(7 + n))
    return got
