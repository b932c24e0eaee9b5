"""Helpers for the tests of the cache in 4 bits."""
from __future__ import annotations

import numpy as np
import torch

from attn_util import normal
from oracle import cache4


def pages4(seed, pages, Hkv, page, D, dtype, unused=None):
    """Pages of normal values: (uint8 tensor, the values). unused [pages, page]: rows that hold NaN."""
    x, x64 = normal(seed, (pages, Hkv, page, D), dtype)
    codes, scales = cache4.quantise(x64, dtype)
    got = cache4.values(codes, scales)
    if unused is not None:
        at = np.broadcast_to(unused[:, None, :, None], scales.shape)
        scales = np.where(at, cache4.NAN, scales).astype(np.uint8)
    return torch.tensor(cache4.pack(codes, scales)), got


def values4(pages, page, D):
    """What pages on the device hold: [n_pages, Hkv, page, D] in fp64."""
    return cache4.values(*cache4.unpack(pages.cpu().numpy(), page, D))
