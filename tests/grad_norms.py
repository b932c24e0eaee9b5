"""How far gradients of attention may be off in their norm.

A gradient is a sum over many products whose factors were rounded, each by at most half a
step: u relative to its value. The roundings are independent, so the squares of what they do
add up, and the mean square of a rounding is a third of the largest one's. gradient_errors
gives, element by element, the root of the sum of the largest squares; a result's error is in
its norm RMS times theirs (1 / sqrt 3, and a tenth for chance and for what is of second order).
An elementwise worst case cannot see that something is missing that changes each element
little; this can."""
from __future__ import annotations

import numpy as np

from oracle import doc_attention as oda

RMS = 1.1 / np.sqrt(3.0)


def gradient_errors(q, k, v, do, sc: oda.Scores, prefix: int, u: float, tiny: float, parts=None, row: float = 0.0):
    """One document: ((dq, dk, dv), (their errors)). dS and P are rounded relative to their values,
    results to the type, whose smallest step is 2 tiny. parts: the output was joined from these slices of
    the keys, each part's rounded and then the whole, and D is do . o of it. row: what a row's log-sum-exp
    is off by, which changes all of its weights alike."""
    rows, H, D = q.shape
    G = H // k.shape[1]
    scale = 1.0 / np.sqrt(D) if sc.scale is None else sc.scale
    d = [np.zeros(x.shape) for x in (q, k, v)]
    e = [np.zeros(x.shape) for x in (q, k, v)]
    for h in range(H):
        g = h // G
        s, t, _ = oda._head(q[:, h], k[:, g], sc, h, prefix)
        p, _ = oda._weights(s)
        dp = do[:, h] @ v[:, g].T
        slip = 1.0 - t * t
        ds = p * (dp - (p * dp).sum(axis=1, keepdims=True)) * slip
        d[0][:, h] = scale * ds @ k[:, g]
        d[1][:, g] += scale * ds.T @ q[:, h]
        d[2][:, g] += p.T @ do[:, h]
        e[0][:, h] = scale ** 2 * ((u * ds) ** 2 @ k[:, g] ** 2)
        e[1][:, g] += scale ** 2 * ((u * ds) ** 2).T @ q[:, h] ** 2
        e[2][:, g] += ((u * p) ** 2).T @ do[:, h] ** 2
        if row:
            e[0][:, h] += (row * d[0][:, h]) ** 2
            e[1][:, g] += scale ** 2 * ((row * ds) ** 2).T @ q[:, h] ** 2
            e[2][:, g] += ((row * p) ** 2).T @ do[:, h] ** 2
        if parts:
            eo = (u * (p @ v[:, g])) ** 2 + (u * p) ** 2 @ v[:, g] ** 2
            for c in parts:
                eo += (u * (p[:, c] @ v[c, g])) ** 2
            ed = (do[:, h] ** 2 * eo).sum(axis=1, keepdims=True)
            e[0][:, h] += ed * (scale * (p * slip) @ k[:, g]) ** 2
            e[1][:, g] += scale ** 2 * (ed * (p * slip) ** 2).T @ q[:, h] ** 2
    return tuple(d), tuple(np.sqrt(y + (u * x) ** 2 + tiny ** 2) for x, y in zip(d, e))


def check_norm(got, want, error, what):
    off, allowed = np.linalg.norm(got - want), RMS * np.linalg.norm(error)
    assert off <= allowed, "%s: off by %.3g of its norm, %.3g allowed" % (what, off / np.linalg.norm(want), allowed / np.linalg.norm(want))


def check_along(got, want, error, slope, what):
    """slope: the derivative along the gradient's own direction, from differences. The errors along it
    add up like the others: four times their root mean square."""
    w = want / np.linalg.norm(want)
    allowed = 4 / np.sqrt(3.0) * np.linalg.norm(error * w) + 1e-6 * abs(slope)
    assert abs((got * w).sum() - slope) <= allowed, "%s: %.6g along the gradient, %.6g by differences" % (what, (got * w).sum(), slope)
