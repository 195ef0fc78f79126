"""The layer operators' entry points and binding at the edges of their arguments, as
far as no device is needed."""
from __future__ import annotations

import ctypes
import types

import pytest
import torch

import paper_2609_00224_amd as q
from tests.test_serving_edges import _cache, calls  # noqa: F401

VP = ctypes.c_void_p
ADDR, OTHER, THIRD = VP(1 << 20), VP(1 << 21), VP(1 << 22)  # never read: no call below launches


def test_sizes_that_the_header_allows_are_not_refused():
    """Rows of 2^29 elements and more: calls that stop, after the checks of their sizes,
    at there being no rows or too small a buffer."""
    lib = q.load()
    for heads, dim in ((65535, 8224), (65535, 65536), (1, 65536)):
        run = heads * dim
        assert lib.qtea_rms_norm(ADDR, 1, run, THIRD, 1, run, None, 0, 1e-6, OTHER, 1, run, None, 0, 0, heads, dim, None) == q.QTEA_OK
        assert lib.qtea_rms_norm(ADDR, 1, run, None, 0, 0, None, 0, 1e-6, OTHER, q.QTEA_E4M3, run, THIRD, run // 32, 0, heads, dim, None) == q.QTEA_OK
    for dim in (2 ** 29, 2 ** 30 + 32, 2 ** 31 - 32):
        assert lib.qtea_silu_mul(ADDR, OTHER, 0, dim, 2 * dim, THIRD, 0, dim, None, 0, 0, dim, None) == q.QTEA_OK
        assert lib.qtea_silu_mul(ADDR, OTHER, 0, dim, 2 * dim, THIRD, q.QTEA_E4M3, dim, ADDR, dim // 32, 0, dim, None) == q.QTEA_OK
    for N in (2 ** 29, 2 ** 30 + 1, 2 ** 31 - 256):
        need = q.qtea_w4_packed_bytes(N, 40)
        assert lib.qtea_w4_gemm_lowbatch(ADDR, need - 1, N, 40, OTHER, 0, 40, None, 0, 3, THIRD, 0, N, None) == q.QTEA_ERR_WORKSPACE


def test_sizes_that_no_grid_or_address_has_are_refused():
    lib, out = q.load(), ctypes.c_int64(0)
    for N in (2 ** 31 - 255, 2 ** 31 - 1):
        assert lib.qtea_w4_packed_bytes(N, 1, ctypes.byref(out)) == q.QTEA_ERR_INVALID_ARG
    for tokens, stride in ((3, 2 ** 38 + 16), (2 ** 31 - 1, 2 ** 29 + 16), (1, 2 ** 62)):
        assert lib.qtea_rms_norm(ADDR, 1, stride, None, 0, 0, None, 0, 1e-6, OTHER, 1, 64, None, 0, tokens, 1, 64, None) == q.QTEA_ERR_INVALID_ARG
        assert lib.qtea_rms_norm(ADDR, 1, 64, None, 0, 0, None, 0, 1e-6, OTHER, 1, stride, None, 0, tokens, 1, 64, None) == q.QTEA_ERR_INVALID_ARG
        assert lib.qtea_silu_mul(ADDR, OTHER, 0, 64, stride, THIRD, 0, 64, None, 0, tokens, 64, None) == q.QTEA_ERR_INVALID_ARG
    assert lib.qtea_w4_gemm_lowbatch(ADDR, 1 << 40, 64, 64, OTHER, 0, 64, None, 0, 3, THIRD, 0, 2 ** 38 + 1, None) == q.QTEA_ERR_INVALID_ARG


class Tensor:
    """Stands for a contiguous device tensor of any shape."""

    def __init__(self, *shape, dtype=torch.float16):
        self.shape, self.dtype = torch.Size(shape), dtype

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def stride(self):
        return tuple(int(torch.Size(self.shape[i + 1:]).numel()) for i in range(len(self.shape)))

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def stream(monkeypatch):
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 1)
    return types.SimpleNamespace(cuda_stream=0)


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32 + 1, 2 ** 33 + 5])
def test_counts_past_the_c_types_range_reach_the_entry_points_check(calls, stream, n):  # noqa: F811
    """They are not taken modulo 2^32: heads, rows of a product, frequencies."""
    q.qtea_rms_norm(Tensor(1, n, 4), None, Tensor(1, n, 4), stream=stream)
    q.qtea_w4_gemm_lowbatch(q.W4Matrix(3, 64, Tensor(5000, dtype=torch.uint8)), Tensor(n, 64), Tensor(n, 3), stream=stream)
    (norm, args), (gemm, margs) = calls.made
    assert norm == "qtea_rms_norm" and ctypes.c_int(args[15]).value >= 65536
    assert gemm == "qtea_w4_gemm_lowbatch" and ctypes.c_int(margs[9]).value > q.QTEA_W4_MAX_BATCH
    calls.made.clear()
    i32 = lambda *s: Tensor(*s, dtype=torch.int32)  # noqa: E731
    k = Tensor(1, 2, 64)
    q.qtea_kv_append_rotated(_cache(device=0), Tensor(1, n, 64), k, k, i32(2), i32(1), i32(1, 5), Tensor(n + 8, dtype=torch.float32), Tensor(1, n, 64), stream=stream)
    (_, args), = calls.made
    assert ctypes.c_int(args[9]).value > 65535 and ctypes.c_int(args[11]).value > 256
