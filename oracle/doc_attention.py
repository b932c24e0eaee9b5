"""Oracle: attention over packed documents with its gradient, and a paged cache, in fp64
(test infrastructure).

Scores of row i and key j of one document, p_i = i + keys - rows:
    s = scale q_i . k_j;  cap c: s = c tanh(s / c);  slope: s -= slope |p_i - j|
Visible keys: all of the document, or j <= p_i or j < prefix. The functions take one
document (or sequence) at a time and write the definition out; the packed forms go through
the documents. Layouts: q, o [rows, H, D], k, v [keys, Hkv, D], lse [H, rows].

`attention_bounds` and the bounds that `attention_grad` returns say how far a result may be
off whose weights (and gradients of scores) are rounded to a type with relative error u and
smallest step `tiny` before they are multiplied, whose products are summed in fp32 and whose
outputs are rounded to the type once. They are first-order worst cases:
    a score:    es = 2^-17 (scale |q| . |k| + |s| + 1): 128 fp32 products summed in any order
                (2^-24 each), and a few roundings of exp2's argument; with a cap c up to 64
                2^-22 c for tanh (beyond, tanh is exact to its own size)
    a weight:   p (2 es + u) + tiny, times |v|, summed
    an output:  u |o| + tiny on top (an fp16 output below 2^-14 is a multiple of 2^-24 too)
    D = do . o: |do| . (u |o| + the bound of o); dP: 2^-17 |do| . |v|
    dS:         |dS| (2 es + u) + p (error of D + error of dP) + tiny
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import numpy as np


class Scores(NamedTuple):
    scale: Optional[float] = None
    cap: float = 0.0
    slopes: Optional[np.ndarray] = None
    causal: bool = True


def visible(rows: int, keys: int, causal: bool, prefix: int = 0) -> np.ndarray:
    p = np.arange(rows)[:, None] + keys - rows
    j = np.arange(keys)[None, :]
    if not causal:
        return np.ones((rows, keys), dtype=bool)
    return (j <= p) | (j < prefix)


def _head(q, k, sc: Scores, h: int, prefix: int):
    """(scores with -inf where masked, tanh of the capped ones, size of the products)."""
    rows, keys = q.shape[0], k.shape[0]
    scale = 1.0 / np.sqrt(q.shape[1]) if sc.scale is None else sc.scale
    s = (q @ k.T) * scale
    size = (np.abs(q) @ np.abs(k).T) * scale
    t = np.zeros_like(s)
    if sc.cap:
        t = np.tanh(s / sc.cap)
        s = sc.cap * t
    if sc.slopes is not None:
        p = np.arange(rows)[:, None] + keys - rows
        d = sc.slopes[h] * np.abs(p - np.arange(keys)[None, :])
        s = s - d
        size = size + d
    size = size + np.abs(s) + 1.0 + min(sc.cap, 64.0) / 32
    return np.where(visible(rows, keys, sc.causal, prefix), s, -np.inf), t, size


# The least normal fp32 number (and bf16 number). Below it a value may count as 0, which it is then off
# by at most: a weight, so that its gradient of a score is off by that times do . v - D, that gradient
# itself, a result.
LEAST = 2.0 ** -126


def _weights(s):
    if s.shape[1] == 0:
        return np.zeros_like(s), np.full(s.shape[0], -np.inf)
    m = s.max(axis=1, keepdims=True)
    m0 = np.where(np.isfinite(m), m, 0.0)
    e = np.exp(s - m0)
    l = e.sum(axis=1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (m0 + np.log(l))[:, 0]
    return e / np.where(l == 0, 1.0, l), lse


def attention(q, k, v, sc: Scores, prefix: int = 0, u: float = 0.0, tiny: float = 0.0):
    """One document: (o, lse, bound of o's error, bound of lse's error)."""
    rows, H, D = q.shape
    G = H // k.shape[1]
    o, lse = np.zeros((rows, H, D)), np.zeros((H, rows))
    eo, el = np.zeros_like(o), np.zeros_like(lse)
    for h in range(H):
        s, _, size = _head(q[:, h], k[:, h // G], sc, h, prefix)
        p, lse[h] = _weights(s)
        vh = v[:, h // G]
        es = 2.0 ** -17 * size
        o[:, h] = p @ vh
        wide = (np.where(p > 0, p * (2 * es + u), 0.0) + (tiny + LEAST) * np.isfinite(s)) @ np.abs(vh)
        eo[:, h] = u * np.abs(o[:, h]) + tiny + LEAST + wide
        el[h] = (p * es).sum(axis=1) + 2.0 ** -20 * (1 + np.abs(np.where(np.isfinite(lse[h]), lse[h], 0.0)))
    return o, lse, eo, el


def attention_grad(q, k, v, do, sc: Scores, prefix: int = 0, u: float = 0.0, tiny: float = 0.0):
    """One document: ((dq, dk, dv), (bounds of their errors))."""
    rows, H, D = q.shape
    G = H // k.shape[1]
    scale = 1.0 / np.sqrt(D) if sc.scale is None else sc.scale
    d = [np.zeros_like(x) for x in (q, k, v)]
    e = [np.zeros_like(x) for x in (q, k, v)]
    o, _, eo, _ = attention(q, k, v, sc, prefix, u, tiny)
    for h in range(H):
        g = h // G
        s, t, size = _head(q[:, h], k[:, g], sc, h, prefix)
        p, _ = _weights(s)
        es = 2.0 ** -17 * size
        seen = np.isfinite(s)
        dp = do[:, h] @ v[:, g].T
        delta = (p * dp).sum(axis=1, keepdims=True)
        slip = 1.0 - t * t
        ds = p * (dp - delta) * slip
        e_delta = (np.abs(do[:, h]) * (eo[:, h] + 2.0 ** -17 * np.abs(o[:, h]))).sum(axis=1, keepdims=True)
        e_dp = 2.0 ** -17 * (np.abs(do[:, h]) @ np.abs(v[:, g]).T)
        e_ds = np.abs(ds) * (2 * es + u) + p * (e_delta + e_dp) + 2.0 ** -20 * p * np.abs(dp - delta) + (tiny + LEAST * (1 + np.abs(dp - delta))) * seen
        e_p = p * (2 * es + u) + (tiny + LEAST) * seen
        d[0][:, h] = scale * ds @ k[:, g]
        e[0][:, h] = scale * e_ds @ np.abs(k[:, g])
        d[1][:, g] += scale * ds.T @ q[:, h]
        e[1][:, g] += scale * e_ds.T @ np.abs(q[:, h])
        d[2][:, g] += p.T @ do[:, h]
        e[2][:, g] += e_p.T @ np.abs(do[:, h])
    for x, b in zip(d, e):
        b += u * np.abs(x) + tiny + LEAST
    return tuple(d), tuple(e)


def rotate(x, positions, inv_freq, interleaved: bool):
    """x [tokens, heads, D] with its first 2 len(inv_freq) elements rotated by position."""
    n = len(inv_freq)
    a = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float64)
    i, j = (2 * np.arange(n), 2 * np.arange(n) + 1) if interleaved else (np.arange(n), np.arange(n) + n)
    y = np.array(x, dtype=np.float64)
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    return y


def cached_rows(pages, table_row, length: int):
    """Tokens 0 .. length - 1 of one sequence: [length, Hkv, D] from [n_pages, Hkv, size, D]."""
    size = pages.shape[2]
    x = np.arange(length)
    return pages[np.asarray(table_row)[x // size], :, x % size]
