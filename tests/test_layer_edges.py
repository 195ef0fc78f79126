"""The layer operators' entry points and binding at the edges of their arguments, as
far as no device is needed."""
from __future__ import annotations

import ctypes

import paper_2609_00224_amd as q

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
