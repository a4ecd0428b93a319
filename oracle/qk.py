"""Oracle of the queries' and keys' treatment in self-attention: the norm per head and the
rotation by the token's place, written out per head and pair.

  norm      y = x / sqrt(mean_d x^2 + eps) * gain
  rotation  pair j of a head belongs to the row axis or the column axis of the patch grid and
            turns by u = place * f: (x cos u - y sin u, x sin u + y cos u), with
            f = theta^(-2 i / dims of the axis) for pair i of the axis
"""
from dataclasses import dataclass

import numpy as np


@dataclass
class QK:
    """q_gain, k_gain: [L, dh] or None (1). dims: head dims of the row and the column axis,
    or None (no rotation). layout: "adjacent", "halves" or "axis_halves"."""
    norm: bool = True
    q_gain: np.ndarray = None
    k_gain: np.ndarray = None
    eps: float = 1e-6
    dims: tuple = None
    theta: float = 10000.0
    layout: str = "adjacent"


def pairs(dims, layout):
    """(first dim, second dim, axis, frequency exponent) of every pair."""
    out, total, base = [], sum(dims) // 2, 0
    for axis, d in enumerate(dims):
        for i in range(d // 2):
            j = base // 2 + i
            if layout == "adjacent":
                lo, hi = 2 * j, 2 * j + 1
            elif layout == "halves":
                lo, hi = j, j + total
            else:
                lo, hi = base + i, base + d // 2 + i
            out.append((lo, hi, axis, -2.0 * i / d))
        base += d
    return out


def treat(x, heads, gain, qk, grid_w):
    """x [N, D] of one sample, token n at place (n // grid_w, n % grid_w)."""
    N, D = x.shape
    dh = D // heads
    y = x.reshape(N, heads, dh)
    if qk.norm:
        y = y / np.sqrt((y * y).mean(axis=-1, keepdims=True) + x.dtype.type(qk.eps))
        if gain is not None:
            y = y * gain.astype(x.dtype)
    if qk.dims is not None:
        out = y.copy()
        n = np.arange(N)
        place = (n // grid_w, n % grid_w)
        for lo, hi, axis, e in pairs(qk.dims, qk.layout):
            u = place[axis] * qk.theta ** e
            c, s = np.cos(u)[:, None].astype(x.dtype), np.sin(u)[:, None].astype(x.dtype)
            out[..., lo] = y[..., lo] * c - y[..., hi] * s
            out[..., hi] = y[..., lo] * s + y[..., hi] * c
        y = out
    return y.reshape(N, D)
