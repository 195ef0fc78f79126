"""What the layer operators' tests share: values of a type, 8-bit rows, bounds."""
from __future__ import annotations

import numpy as np
import torch

import oracle.serving as sv
from tests.serving_cases import TORCH, rounded  # noqa: F401

HALF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # relative half steps
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -150}  # half of the smallest step
U = 2.0 ** -24


def room(shape, kind, device="cuda"):
    """An output of that type (8 bits: codes, scales), filled with a mark."""
    if kind != "e4m3":
        return torch.full(shape, 7.0, dtype=TORCH[kind], device=device), None
    return (torch.full(shape, 0x55, dtype=torch.uint8, device=device),
            torch.full((*shape[:-1], shape[-1] // 32), 0x55, dtype=torch.uint8, device=device))


def values(out, scale):
    """An output's values, fp64 on the host."""
    if scale is None:
        return out.double().cpu().numpy()
    return sv.decode(out.cpu().numpy(), scale.cpu().numpy(), "e4m3")


def check(out, scale, want, kind, err, what=""):
    """The output is `want` (fp64), off by at most `err` (an array, what the
    fp32 arithmetic before the last rounding may be off) and that rounding.

    8 bits: the block's scale is the rule's for some values within err of
    want's; a code is off by half a step: 2^-4 of the value, or 2^-10 of the
    block's unit below the smallest normal code."""
    err = np.broadcast_to(err, want.shape)
    got = values(out, scale)
    if kind != "e4m3":
        bound = err + HALF[kind] * (np.abs(want) + err) + TINY[kind]
    else:
        e = scale.cpu().numpy().astype(int) - 127
        blocks = lambda v: v.reshape(*v.shape[:-1], -1, 32)  # noqa: E731
        most, least = blocks(np.abs(want) + err).max(-1), blocks(np.abs(want) - err).max(-1)
        assert ((least <= 448 * 2.0 ** e) | (e == 7)).all() and ((most > 224 * 2.0 ** e) | (e == -15)).all(), what
        unit = np.repeat(2.0 ** e, 32, -1).reshape(want.shape)
        want = np.clip(want, -448 * unit, 448 * unit)
        bound = err + 2.0 ** -4 * (np.abs(want) + err) + 2.0 ** -10 * unit
    off = np.abs(got - want)
    worst = np.unravel_index(np.argmax(off - bound), off.shape)
    assert (off <= bound).all(), f"{what}: {got[worst]} for {want[worst]}, off by {off[worst]} of {bound[worst]} at {worst}"
