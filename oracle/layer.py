"""Plain definitions of a decoder layer's row operators in numpy, fp64 (angles
in extended precision): the norm with the residual's addition, the gated
activation, the rotation by position, products with 4-bit codes.  Shares no code
with the library or its binding; the block formats are oracle.serving's.
"""
from __future__ import annotations

import numpy as np

from . import serving as sv


def rms_norm(x, weight, eps, residual=None):
    """Rows x [..., dim] fp64: (out, t) with t = x + residual."""
    t = x if residual is None else x + residual
    y = t / np.sqrt((t * t).mean(-1, keepdims=True) + eps)
    return (y if weight is None else y * weight), t


def silu_mul(gate, up):
    with np.errstate(over="ignore"):
        return gate / (1.0 + np.exp(-gate)) * up


def rotate(x, positions, freq, interleaved=False):
    """x [n][heads][dim] fp64 at `positions` [n], freq fp32 [rot / 2]."""
    half = len(freq)
    angle = np.asarray(positions, np.longdouble)[:, None] * np.asarray(freq, np.longdouble)  # exact: 31 + 24 of 64 bits
    cos, sin = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
    a, b = (np.arange(half) * 2, np.arange(half) * 2 + 1) if interleaved else (np.arange(half), np.arange(half) + half)
    out = np.array(x, np.float64)
    out[..., a], out[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    return out


def w4_values(W):
    """The values that a matrix W [N][K] fp64 has in blocks of 32 E2M1 codes."""
    N, K = W.shape
    padded = np.zeros((N, -(-K // 32) * 32))
    padded[:, :K] = W
    return sv.decode(*sv.encode(padded, "e2m1"), "e2m1")[:, :K]
