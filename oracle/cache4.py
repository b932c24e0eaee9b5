"""Oracle: elements in 4 bits with a scale per 32 (OCP MXFP4), in fp64 (test infrastructure).

A block of 32 elements has scale 2^(byte - 127) and elements (-1)^(code / 8) GRID[code % 8] times
it. The scale is the least of the type's range with no element beyond 7 times it; an element is
the nearest value of the grid, of two equally near the one with the even code. A block that is
not finite has byte 255 and stands for NaN.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LIMITS = {"bf16": (2, 252), "f16": (104, 140)}  # of the byte
NAN = 255


def quantise(x, dtype: str):
    """x [..., D] in fp64: (codes [..., D], bytes [..., D / 32])."""
    x = np.asarray(x, dtype=np.float64)
    y = x.reshape(x.shape[:-1] + (-1, 32))
    top = np.abs(y).max(axis=-1)
    bad = ~np.isfinite(y).all(axis=-1)
    lo, hi = LIMITS[dtype]
    byte = np.full(top.shape, lo)
    for b in range(lo, hi):
        byte[~bad & (top > 7.0 * 2.0 ** (b - 127))] = b + 1
    z = np.where(bad[..., None], 0.0, y) / 2.0 ** (byte[..., None] - 127.0)
    off = np.abs(np.abs(z)[..., None] - GRID)
    near = off == off.min(axis=-1, keepdims=True)
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(axis=-1), even.argmax(axis=-1), near.argmax(axis=-1)) + 8 * (z < 0)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, NAN, byte).astype(np.uint8)


def values(codes, scales):
    """What codes [..., D] and scales [..., D / 32] stand for."""
    x = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == NAN, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    return x * np.repeat(s, 32, axis=-1)


def pack(codes, scales):
    """Pages [n_pages, Hkv, size * (D / 2 + D / 32)] from [n_pages, Hkv, size, D] and [n_pages, Hkv, size, D / 32]."""
    both = codes[..., 0::2] | codes[..., 1::2] << 4
    return np.concatenate([x.reshape(x.shape[:2] + (-1,)) for x in (both, scales)], axis=-1).astype(np.uint8)


def unpack(pages, size: int, d: int):
    """The reverse: (codes, scales)."""
    both = pages[..., :size * d // 2].reshape(pages.shape[:2] + (size, d // 2))
    codes = np.stack([both & 15, both >> 4], axis=-1).reshape(pages.shape[:2] + (size, d))
    return codes, pages[..., size * d // 2:].reshape(pages.shape[:2] + (size, d // 32))
