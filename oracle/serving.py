"""Plain definitions of the serving operators in numpy, fp64 and whole numbers.

The cache format, attention over it and the verification of drafts, written
from their formulas for one sequence and one head at a time.  Shares no code
with the library or its binding.
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])
LADDER = {"e4m3": E4M3, "e2m1": E2M1}
EXPONENTS = {"e4m3": (-15, 7), "e2m1": (-23, 13)}
BLOCK = 32


def encode(x, fmt):
    """x [..., dim] fp64 (values of fp32 or fewer bits): (code values' indices
    with the sign in bit 7 (E4M3) or 3 (E2M1), scale bytes).  A block's scale is
    the smallest power of two under which its largest magnitude is at most the
    largest code; a block with a NaN or an infinity has scale 255."""
    ladder, (low, high) = LADDER[fmt], EXPONENTS[fmt]
    b = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, BLOCK)
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    amax = np.abs(b).max(-1)
    units = 2.0 ** np.arange(low, high + 1)
    e = np.minimum(np.searchsorted(units * ladder[-1], amax), len(units) - 1)
    a = np.minimum(np.abs(b) / units[e][..., None], ladder[-1])
    mid = (ladder[1:] + ladder[:-1]) / 2
    lo, hi = np.searchsorted(mid, a, side="left"), np.searchsorted(mid, a, side="right")
    code = np.where(lo % 2 == 0, lo, hi).astype(np.uint8)  # on a tie the even code
    code |= np.where(np.signbit(b), 128 if fmt == "e4m3" else 8, 0).astype(np.uint8)
    scale = np.where(bad, 255, e + low + 127).astype(np.uint8)
    return code.reshape(x.shape), scale


def decode(code, scale, fmt):
    """The values of encode's result (NaN for a block of scale 255)."""
    mask = 127 if fmt == "e4m3" else 7
    ladder = np.append(LADDER[fmt], np.nan)
    v = ladder[np.minimum(code & mask, len(ladder) - 1)] * np.where(code > mask, -1.0, 1.0)
    b = v.reshape(*v.shape[:-1], -1, BLOCK)
    unit = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return (b * unit[..., None]).reshape(v.shape)


def attention(q, k, v, positions, scale, window=0):
    """One head: rows q [n][dim] at `positions` over k, v [len][dim] (fp64).
    Returns (out, spread): spread is the weights' mean of |v|."""
    out, spread = np.zeros_like(q), np.zeros_like(q)
    for i, p in enumerate(positions):
        lo = max(0, p + 1 - window) if window else 0
        if p < 0:
            continue
        s = (k[lo:p + 1] @ q[i]) * scale
        w = np.exp(s - s.max())
        w /= w.sum()
        out[i], spread[i] = w @ v[lo:p + 1], w @ np.abs(v[lo:p + 1])
    return out, spread


def _units(p, bits):
    """floor(2^bits p), p limited to [0, 1] (NaN: 0)."""
    if not p > 0:
        return 0
    return int(Fraction(min(float(p), 1.0)) * (1 << bits))


def verify(target, draft, tokens, u_accept, u_sample):
    """One sequence: target [n + 1][vocab], draft [n][vocab] (None: all of a
    draft's mass on its token), tokens and u_accept [n].  Returns (accepted,
    next token)."""
    n, vocab = len(tokens), target.shape[1]
    for i in range(n + 1):
        P = [_units(p, 38) for p in target[i]]
        Q = [0] * vocab
        if i < n:
            x = int(tokens[i])
            if draft is not None:
                Q = [_units(p, 38) for p in draft[i]]
            elif 0 <= x < vocab:
                Q[x] = 1 << 38
            u = min(_units(u_accept[i], 24), (1 << 24) - 1)
            if 0 <= x < vocab and u * Q[x] < P[x] << 24:
                continue
        W = [max(a - b, 0) for a, b in zip(P, Q)]
        if sum(W) == 0:
            W = P
        r = (min(_units(u_sample, 24), (1 << 24) - 1) * sum(W)) >> 24
        c = 0
        for t, w in enumerate(W):
            c += w
            if c > r:
                return i, t
        return i, -1
