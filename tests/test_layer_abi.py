"""Host-side checks of the layer entry points (include/qtea_layer.h) and of
qtea_kv_append_rotated: what they refuse, before anything reaches a device;
and the oracle's definitions by hand."""
from __future__ import annotations

import ctypes
import os

import numpy as np
import pytest
import torch

import oracle.layer as ol
import paper_2609_00224_amd as q
from tests.test_serving_abi import BAD_BATCHES, BAD_CACHES, _batch, _cache

VP = ctypes.c_void_p
ADDR, OTHER, THIRD = VP(1 << 20), VP(1 << 21), VP(1 << 22)  # never read: every call below is refused
ODD = VP((1 << 20) + 1)
BAD = q.QTEA_ERR_INVALID_ARG


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(q.LIB_PATH):
        pytest.fail("libqtea.so is not built: run __graft_entry__.build()")
    return q.load()


def test_norm_refuses(lib):
    def call(x=ADDR, xt=2, xs=64, r=None, rt=0, rs=64, w=None, wt=0, eps=1e-6, out=OTHER, ot=0, os_=64, sc=None, ss=0, tokens=3, heads=1, dim=64):
        return lib.qtea_rms_norm(x, xt, xs, r, rt, rs, w, wt, eps, out, ot, os_, sc, ss, tokens, heads, dim, None)

    for change in (dict(x=None), dict(out=None), dict(xt=3), dict(xt=-1), dict(xs=63), dict(xs=1 << 40), dict(x=VP((1 << 20) + 2)), dict(ot=4), dict(ot=-1),
                   dict(os_=63), dict(out=VP((1 << 21) + 1)), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-40),
                   dict(r=THIRD, rt=3), dict(r=THIRD, rs=63), dict(r=VP((1 << 22) + 1)), dict(r=ADDR), dict(r=OTHER), dict(w=THIRD, wt=3), dict(w=VP((1 << 22) + 1)),
                   dict(w=OTHER), dict(tokens=-1), dict(tokens=1 << 31), dict(heads=0), dict(heads=65536), dict(heads=2), dict(dim=0), dict(dim=65537, xs=65537, os_=65537),
                   dict(sc=THIRD), dict(ot=3), dict(ot=3, sc=THIRD, ss=1), dict(ot=3, sc=THIRD, ss=2, os_=72), dict(ot=3, sc=THIRD, ss=2, out=VP((1 << 21) + 8)),
                   dict(ot=3, sc=THIRD, ss=2, dim=48), dict(x=OTHER, xt=2, ot=0), dict(x=OTHER, xt=0, ot=0, xs=72)):
        assert call(**change) == BAD, change
    assert call(tokens=0) == q.QTEA_OK


def test_gate_refuses(lib):
    def call(g=ADDR, u=OTHER, t=2, gs=64, us=64, out=THIRD, ot=0, os_=64, sc=None, ss=0, rows=3, dim=64):
        return lib.qtea_silu_mul(g, u, t, gs, us, out, ot, os_, sc, ss, rows, dim, None)

    for change in (dict(g=None), dict(u=None), dict(out=None), dict(t=3), dict(t=-1), dict(gs=63), dict(us=63), dict(g=ODD), dict(u=ODD), dict(out=ODD), dict(ot=4),
                   dict(os_=63), dict(rows=-1), dict(rows=1 << 31), dict(dim=0), dict(rows=1 << 30), dict(sc=ADDR), dict(ot=3), dict(ot=3, sc=ADDR, ss=2, dim=40),
                   dict(out=ADDR, ot=0), dict(out=OTHER, ot=2, os_=72)):
        assert call(**change) == BAD, change
    assert call(rows=0) == q.QTEA_OK


def test_w4_refuses(lib):
    need = q.qtea_w4_packed_bytes(100, 96)

    def gemm(p=ADDR, nbytes=need, N=100, K=96, X=OTHER, xt=0, xs=96, sc=None, ss=0, batch=3, Y=THIRD, yt=2, ys=100):
        return lib.qtea_w4_gemm_lowbatch(p, nbytes, N, K, X, xt, xs, sc, ss, batch, Y, yt, ys, None)

    for change in (dict(p=None), dict(X=None), dict(Y=None), dict(p=VP((1 << 20) + 8)), dict(N=0), dict(K=0), dict(N=1 << 31), dict(K=(1 << 24) + 1), dict(xt=2), dict(xt=4),
                   dict(xs=95), dict(xs=1 << 29), dict(xt=3, sc=ADDR, ss=1 << 30), dict(X=ODD), dict(Y=ODD), dict(yt=3), dict(ys=99), dict(sc=ADDR), dict(xt=3), dict(xt=3, sc=ADDR, ss=2), dict(xt=3, sc=ADDR, ss=3, xs=104),
                   dict(xt=3, sc=ADDR, ss=3, X=VP((1 << 21) + 8)), dict(xt=3, sc=ADDR, ss=3, K=90)):
        assert gemm(**change) == BAD, change
    assert gemm(batch=0) == gemm(batch=65) == q.QTEA_ERR_BATCH
    assert gemm(nbytes=need - 1) == q.QTEA_ERR_WORKSPACE
    for name in ("qtea_w4_pack", "qtea_w4_unpack"):
        def call(W=ADDR, t=0, ws=96, N=100, K=96, p=OTHER, nbytes=need):
            args = (W, t, ws, N, K, p, nbytes) if name == "qtea_w4_pack" else (p, nbytes, N, K, W, t, ws)
            return getattr(lib, name)(*args, None)

        for change in (dict(W=None), dict(p=None), dict(t=3), dict(t=-1), dict(ws=95), dict(W=ODD), dict(p=VP((1 << 20) + 8)), dict(N=0), dict(K=0), dict(N=1 << 31)):
            assert call(**change) == BAD, change
        assert call(nbytes=need - 1) == q.QTEA_ERR_WORKSPACE
    out = ctypes.c_int64(0)
    assert lib.qtea_w4_packed_bytes(1, 1, None) == BAD and lib.qtea_w4_packed_bytes(0, 1, ctypes.byref(out)) == BAD
    # 4.25 bits a weight where tiles are full
    assert q.qtea_w4_packed_bytes(1024, 2048) == 1024 * 2048 * 17 // 32


def test_rotated_append_refuses(lib):
    def call(cache=None, batch=None, Q=THIRD, k=ADDR, v=ADDR, t=2, qs=256, ks=128, vs=128, heads=4, freq=ADDR, rot=64, out=OTHER, ot=0, os_=256):
        return lib.qtea_kv_append_rotated(cache or _cache(), batch or _batch(), Q, k, v, t, qs, ks, vs, heads, freq, rot, 0, out, ot, os_, None)

    for change in BAD_CACHES:
        assert call(cache=_cache(**change)) == BAD, change
    for change in BAD_BATCHES:
        assert call(batch=_batch(**change)) == BAD, change
    for change in (dict(Q=None), dict(k=None), dict(v=None), dict(out=None), dict(freq=None), dict(freq=VP((1 << 20) + 2)), dict(t=3), dict(qs=255), dict(qs=258), dict(ks=127),
                   dict(vs=130), dict(os_=255), dict(os_=260), dict(Q=VP((1 << 22) + 8)), dict(out=VP((1 << 21) + 8)), dict(ot=3), dict(ot=-1), dict(heads=-1),
                   dict(heads=65536), dict(rot=0), dict(rot=24), dict(rot=80), dict(rot=-16), dict(Q=OTHER), dict(Q=OTHER, ot=2, os_=512)):
        assert call(**change) == BAD, change
    assert call(batch=_batch(n_tokens=0)) == q.QTEA_OK


def test_the_binding_refuses():
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    for call in (lambda: q.qtea_rms_norm(z(2, 64), None, z(2, 64)),  # host tensors
                 lambda: q.qtea_silu_mul(z(2, 64), z(2, 64), z(2, 64)),
                 lambda: q.qtea_w4_gemm_lowbatch(q.W4Matrix(3, 64, z(64, dt=torch.uint8)), z(2, 64), z(2, 3)),
                 lambda: q.qtea_w4_gemm_lowbatch(q.W4Matrix(3, 64, z(64, dt=torch.uint8)), z(2, 65), z(2, 3)),
                 lambda: q.qtea_w4_pack(z(3, 64), z(5000, dt=torch.uint8)),
                 lambda: q.qtea_w4_pack(z(64, 3).T, z(5000, dt=torch.uint8))):
        with pytest.raises(ValueError):
            call()


def test_oracle_by_hand():
    y, t = ol.rms_norm(np.array([[1.0, 2.0]]), np.array([1.0, 10.0]), 0.5, np.array([[0.0, 1.0]]))
    assert np.allclose(t, [[1, 3]]) and np.allclose(y, [[1 / 5.5 ** 0.5, 30 / 5.5 ** 0.5]])
    assert np.allclose(ol.silu_mul(np.array([0.0, 1.0, -1000.0]), np.array([3.0, 2.0, 1.0])), [0, 2 / (1 + np.exp(-1)), 0])
    x = np.arange(6.0).reshape(1, 1, 6)
    quarter = np.float32([np.pi / 2, 0])
    assert np.allclose(ol.rotate(x, [1], quarter), [[[-2, 1, 0, 3, 4, 5]]], atol=1e-6)
    assert np.allclose(ol.rotate(x, [1], quarter, True), [[[-1, 0, 2, 3, 4, 5]]], atol=1e-6)
    assert np.array_equal(ol.w4_values(np.array([[6.0, 0.3, -5.0]])), [[6, 0.5, -4]])  # a tie goes to the even code


def test_the_binding_checks_shapes_before_devices_are_asked_for():
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    m = q.W4Matrix(3, 64, z(64, dt=torch.uint8))
    for call in (lambda: q.qtea_w4_gemm_lowbatch(m, z(64), z(3)), lambda: q.qtea_w4_gemm_lowbatch(m, z(2, 1, 64), z(2, 1, 3)),
                 lambda: q.qtea_w4_gemm_lowbatch(m, z(2, 64), z(3, 3)), lambda: q.qtea_rms_norm(z(64), None, z(64)),
                 lambda: q.qtea_w4_unpack(m, z(3, 64))):
        with pytest.raises(ValueError):
            call()
