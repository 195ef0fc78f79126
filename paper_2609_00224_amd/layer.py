"""Operators of a decoder layer of libqtea.so (include/qtea_layer.h): the
root-mean-square norm with the residual's addition, the gated activation, and
products with matrices of 4-bit codes.

As the rest of the binding, these functions marshal arguments only; every step
runs in the kernels of ``csrc/layer.hip`` and ``csrc/w4.hip``.  They are exported
by the package itself, which imports this module when the first of them is
asked for.

8-bit rows (outputs of the norm and the activation, a product's activations)
are two tensors: uint8 E4M3 codes [rows][n], and uint8 scale bytes [rows][n / 32],
a block of 32 codes standing for code * 2^(scale - 127).
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

import paper_2609_00224_amd as _q
from paper_2609_00224_amd import QTEA_E4M3
from paper_2609_00224_amd.serving import _TYPES, _call, _int, _type

_U8 = torch.uint8


def _tokens(t, run, what, device):
    """A dense operand, [tokens][dim] or [tokens][heads][dim], whose tokens are
    `run` elements, contiguous: the stride of its tokens (of one token it is not
    used, whatever the view has)."""
    if t.get_device() != device:
        raise ValueError(f"{what}: a device tensor, a call's of one device")
    if t.is_contiguous():
        return run
    shape, stride = t.shape, t.stride()
    if len(shape) == 2:
        if stride[1] != 1 and shape[1] > 1:
            raise ValueError(f"{what}: a row's elements are contiguous")
    elif (stride[2] != 1 and shape[2] > 1) or (stride[1] != shape[2] and shape[1] > 1):
        raise ValueError(f"{what}: a token's heads and elements are contiguous")
    return stride[0] if shape[0] > 1 else run


def _scales(codes, scale, run, what):
    """The scale bytes of 8-bit rows: their address and row stride."""
    if scale is None or scale.dtype is not _U8 or tuple(scale.shape) != (*codes.shape[:-1], codes.shape[-1] // 32):
        raise ValueError(f"{what}: uint8, one for each 32 codes of a row")
    return scale.data_ptr(), _tokens(scale, run // 32, what, codes.get_device())


def _out(out, out_scale, run, device):
    """An output's type, stride, scales and their stride."""
    stride, kind = _tokens(out, run, "out", device), _TYPES.get(out.dtype)
    if kind is not None:
        if out_scale is not None:
            raise ValueError("out_scale: for 8-bit outputs only")
        return kind, stride, None, 0
    if out.dtype is not _U8:
        raise ValueError(f"out: fp16, bf16, fp32 or uint8 codes, got {out.dtype}")
    if out.shape[-1] % 32:
        raise ValueError("out: 8-bit rows are a multiple of 32 long")
    return QTEA_E4M3, stride, *_scales(out, out_scale, run, "out_scale")


def qtea_rms_norm(x, weight, out, residual=None, eps: float = 1e-6, out_scale=None, stream=None):
    """out = t / sqrt(mean(t^2) + eps) * weight with t = x + residual, which also
    becomes the residual's new value.  x, out and residual: [rows][dim], or
    [tokens][heads][dim] with a norm per head (fp16, bf16 or fp32 each, rows
    of any stride; out may be x); weight [dim] or None.  out may also be uint8
    E4M3 codes, with out_scale."""
    shape, dev = x.shape, x.get_device()
    if dev < 0:
        raise ValueError("qtea entry points take device tensors")
    heads = 1 if len(shape) == 2 else (shape[1] if len(shape) == 3 else 0)
    if heads == 0 or out.shape != shape or (residual is not None and residual.shape != shape):
        raise ValueError("x, out and residual: one shape, [rows][dim] or [tokens][heads][dim]")
    run = heads * shape[-1]
    xs = _tokens(x, run, "x", dev)
    rs, rt, rp = (0, 0, None) if residual is None else (_tokens(residual, run, "residual", dev), _type(residual, "residual"), residual.data_ptr())
    wt, wp = 0, None
    if weight is not None:
        if weight.shape != shape[-1:] or not weight.is_contiguous() or weight.get_device() != dev:
            raise ValueError("weight: contiguous [dim] of x's device")
        wt, wp = _type(weight, "weight"), weight.data_ptr()
    kind, os_, sp, ss = _out(out, out_scale, run, dev)
    if 0 in shape:
        return
    _call("qtea_rms_norm", dev, stream, x.data_ptr(), _type(x, "x"), xs, rp, rt, rs, wp, wt, eps, out.data_ptr(), kind, os_, sp, ss,
          shape[0], _int(heads), shape[-1])


def qtea_silu_mul(gate, up, out, out_scale=None, stream=None):
    """out = gate / (1 + exp(-gate)) * up; all [rows][dim] (gate and up of one
    type, fp16, bf16 or fp32; rows of any stride; out may be either of them).
    out may also be uint8 E4M3 codes, with out_scale."""
    dev = gate.get_device()
    if dev < 0:
        raise ValueError("qtea entry points take device tensors")
    shape = gate.shape
    if len(shape) != 2 or up.shape != shape or out.shape != shape or up.dtype is not gate.dtype:
        raise ValueError("gate, up and out: one shape [rows][dim], gate and up one type")
    rows, dim = shape
    gs, us = _tokens(gate, dim, "gate", dev), _tokens(up, dim, "up", dev)
    kind, os_, sp, ss = _out(out, out_scale, dim, dev)
    if rows == 0 or dim == 0:
        return
    _call("qtea_silu_mul", dev, stream, gate.data_ptr(), up.data_ptr(), _type(gate, "gate and up"), gs, us, out.data_ptr(), kind, os_, sp, ss, rows, dim)


# ---------------------------------------------------------------------------
# Matrices of 4-bit codes.
# ---------------------------------------------------------------------------
@dataclass
class W4Matrix:
    """A matrix [N][K] in blocks of 32 E2M1 codes with a power of two each."""
    N: int
    K: int
    packed: object  # torch uint8 device tensor


def qtea_w4_packed_bytes(N: int, K: int) -> int:
    out = ctypes.c_int64(0)
    _q._check(_q.load().qtea_w4_packed_bytes(N, K, ctypes.byref(out)), "qtea_w4_packed_bytes")
    return out.value


def _dense(W, packed):
    if W.dim() != 2 or (W.stride(1) != 1 and W.shape[1] > 1):
        raise ValueError("W: [N][K], a row contiguous")
    if W.get_device() < 0 or packed.get_device() != W.get_device() or not packed.is_contiguous():
        raise ValueError("W and packed: tensors of one device, packed contiguous")
    return W.shape[1] if W.shape[0] <= 1 else W.stride(0)


def qtea_w4_pack(W, packed, stream=None):
    """Pack W [N][K] (fp16, bf16 or fp32, rows of any stride) into `packed`
    (uint8, >= qtea_w4_packed_bytes(N, K))."""
    stride = _dense(W, packed)
    _call("qtea_w4_pack", W.get_device(), stream, W.data_ptr(), _type(W, "W"), stride, *W.shape, packed.data_ptr(), packed.numel() * packed.element_size())


def qtea_w4_unpack(matrix: W4Matrix, W, stream=None):
    """The values that a packed matrix stands for, into W [N][K] (exact in
    fp16, bf16 and fp32)."""
    packed = matrix.packed
    stride = _dense(W, packed)
    if tuple(W.shape) != (matrix.N, matrix.K):
        raise ValueError(f"W: [{matrix.N}][{matrix.K}]")
    _call("qtea_w4_unpack", W.get_device(), stream, packed.data_ptr(), packed.numel() * packed.element_size(), *W.shape, W.data_ptr(), _type(W, "W"), stride)


def pack_matrix_w4(W, stream=None) -> W4Matrix:
    """Allocate the packed buffer and pack."""
    packed = torch.empty(qtea_w4_packed_bytes(*W.shape), dtype=_U8, device=W.device)
    qtea_w4_pack(W, packed, stream=stream)
    return W4Matrix(W.shape[0], W.shape[1], packed)


def qtea_w4_gemm_lowbatch(matrix: W4Matrix, X, Y, x_scale=None, stream=None):
    """Y = X W^T: X [rows][K] fp16 or bf16, or uint8 E4M3 codes with x_scale; Y
    [rows][N] fp16, bf16 or fp32; up to QTEA_W4_MAX_BATCH rows of any stride."""
    packed, dev, N, K = matrix.packed, X.get_device(), matrix.N, matrix.K
    rows = X.shape[0]
    if tuple(X.shape) != (rows, K) or tuple(Y.shape) != (rows, N):
        raise ValueError(f"X: [rows][{K}], Y: [rows][{N}]")
    if dev < 0 or packed.get_device() != dev or not packed.is_contiguous():
        raise ValueError("X and the matrix: tensors of one device")
    xs, ys = _tokens(X, K, "X", dev), _tokens(Y, N, "Y", dev)
    if X.dtype is _U8:
        kind, (sp, ss) = QTEA_E4M3, _scales(X, x_scale, K, "x_scale")
    else:
        kind, sp, ss = _type(X, "X"), None, 0
        if x_scale is not None:
            raise ValueError("x_scale: for 8-bit rows only")
    if rows == 0:
        return
    _call("qtea_w4_gemm_lowbatch", dev, stream, packed.data_ptr(), packed.numel() * packed.element_size(), N, K, X.data_ptr(), kind, xs,
          sp, ss, _int(rows), Y.data_ptr(), _type(Y, "Y"), ys)
