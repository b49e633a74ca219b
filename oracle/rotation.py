"""Norm of each head and rotation by position, the plain definition (fp64, CPU), and its gradients.

TEST INFRASTRUCTURE ONLY, like the rest of this package.

For a row x of D values at position p:  n = gamma x / sqrt(mean(x^2) + eps)  (gamma None: n = x);  the pairs (a, b) among the first `rot`
values of n are turned by p * inv_freq[i]:  a' = a cos - b sin,  b' = a sin + b cos.  Pair i is (i, i + rot / 2), or (2i, 2i + 1) where
`interleaved` is set.

Pins (tests/test_oracle_rotation.py): lengths of pairs and the norm, dot products that depend on the distance of positions alone, a hand
example, central differences of the forward function for every gradient.
"""
from __future__ import annotations

import numpy as np


def pairs(rot: int, interleaved: bool):
    """Indices of the a and the b of every pair."""
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def turn(x, positions, inv_freq, rot: int, interleaved: bool, back: bool = False):
    """x [tokens, heads, D] -> turned (back: by the opposite angles)."""
    y = np.array(x, dtype=np.float64)
    if rot == 0:
        return y
    a, b = pairs(rot, interleaved)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float64)[None, :]
    c, s = np.cos(angle)[:, None, :], np.sin(angle)[:, None, :] * (-1.0 if back else 1.0)
    xa, xb = y[..., a].copy(), y[..., b].copy()
    y[..., a] = xa * c - xb * s
    y[..., b] = xa * s + xb * c
    return y


def norm_rotate(x, gamma, positions, inv_freq, rot: int, interleaved: bool, eps: float):
    x = np.asarray(x, dtype=np.float64)
    if gamma is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gamma, dtype=np.float64)
    return turn(x, positions, inv_freq, rot, interleaved)


def norm_rotate_bwd(x, gamma, positions, inv_freq, rot: int, interleaved: bool, eps: float, dy):
    """(dx, dgamma) of norm_rotate for the upstream gradient dy; dgamma None without a norm."""
    x = np.asarray(x, dtype=np.float64)
    z = turn(dy, positions, inv_freq, rot, interleaved, back=True)
    if gamma is None:
        return z, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u = z * np.asarray(gamma, dtype=np.float64)
    return r * (u - x * r * r * (u * x).mean(-1, keepdims=True)), (z * x * r).sum((0, 1))


def pair_sizes(x, rot: int, interleaved: bool):
    """For every value the length of the pair it is in (itself where it does not turn): what its rounding errors are measured by."""
    y = np.abs(np.array(x, dtype=np.float64))
    if rot:
        a, b = pairs(rot, interleaved)
        y[..., a] = y[..., b] = np.hypot(y[..., a], y[..., b])
    return y
