"""Host-side checks of the serving entry points (include/qtea_serve.h): what
they refuse, before anything reaches a device; and the oracle's format."""
from __future__ import annotations

import ctypes
import os

import numpy as np
import pytest
import torch

import oracle.serving as sv
import paper_2609_00224_amd as q

VP = ctypes.c_void_p
ADDR = VP(1 << 20)  # never read: every call below is refused


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(q.LIB_PATH):
        pytest.fail("libqtea.so is not built: run __graft_entry__.build()")
    return q.load()


def _cache(**change):
    f = dict(k=1 << 20, v=1 << 20, k_scale=1 << 20, v_scale=1 << 20, n_pages=4, format=2, n_heads=2, head_dim=64, page_size=16)
    return q.QteaKvCache(**{**f, **change})


def _batch(**change):
    f = dict(q_start=1 << 20, kv_len=1 << 20, page_table=1 << 20, n_tokens=3, n_seq=2, max_pages=5)
    return q.QteaKvBatch(**{**f, **change})


BAD_CACHES = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=(1 << 20) + 8), dict(n_pages=0), dict(n_pages=1 << 31),
              dict(format=-1), dict(format=4), dict(n_heads=0), dict(head_dim=0), dict(head_dim=48), dict(head_dim=288),
              dict(page_size=8), dict(page_size=48), dict(page_size=8192)]
BAD_BATCHES = [dict(q_start=None), dict(kv_len=None), dict(page_table=None), dict(n_tokens=-1), dict(n_tokens=1 << 31), dict(n_seq=0),
               dict(max_pages=0), dict(max_pages=1 << 28)]


def test_the_structures_are_the_headers(lib):
    assert ctypes.sizeof(q.QteaKvCache) == 56 and q.QteaKvCache.format.offset == 40
    assert ctypes.sizeof(q.QteaKvBatch) == 40 and q.QteaKvBatch.n_seq.offset == 32


@pytest.mark.parametrize("name", ["qtea_kv_append", "qtea_kv_read"])
def test_cache_writes_and_reads_refuse(lib, name):
    def call(cache=None, batch=None, k=ADDR, v=ADDR, type=2, ks=128, vs=128):
        return getattr(lib, name)(cache or _cache(), batch or _batch(), k, v, type, ks, vs, None)

    bad = q.QTEA_ERR_INVALID_ARG
    assert getattr(lib, name)(None, _batch(), ADDR, ADDR, 2, 128, 128, None) == bad
    assert getattr(lib, name)(_cache(), None, ADDR, ADDR, 2, 128, 128, None) == bad
    for change in BAD_CACHES:
        assert call(cache=_cache(**change)) == bad, change
    for change in BAD_BATCHES:
        assert call(batch=_batch(**change)) == bad, change
    for change in (dict(k=None), dict(v=None), dict(k=VP((1 << 20) + 4)), dict(type=3), dict(type=-1), dict(ks=127), dict(vs=127),
                   dict(ks=130), dict(type=0, ks=132), dict(vs=1 << 62)):
        assert call(**change) == bad, change
    assert call(batch=_batch(n_tokens=0)) == q.QTEA_OK  # nothing to do


def test_attention_refuses(lib):
    need = 1 << 40

    def call(cache=None, batch=None, Q=ADDR, out=ADDR, type=0, heads=8, qs=512, os_=512, scale=0.1, window=0, ws=ADDR, nbytes=need):
        return lib.qtea_paged_attention(cache or _cache(), batch or _batch(), Q, out, type, heads, qs, os_, scale, window, ws, nbytes, None)

    bad = q.QTEA_ERR_INVALID_ARG
    for change in BAD_CACHES:
        assert call(cache=_cache(**change)) == bad, change
    for change in BAD_BATCHES:
        assert call(batch=_batch(**change)) == bad, change
    for change in (dict(Q=None), dict(out=None), dict(ws=None), dict(Q=VP((1 << 20) + 2)), dict(ws=VP((1 << 20) + 4)), dict(type=2), dict(type=-1),
                   dict(heads=0), dict(heads=1), dict(heads=5), dict(heads=65536), dict(qs=511), dict(os_=511), dict(qs=516), dict(os_=514),
                   dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1),
                   dict(cache=_cache(format=0, k_scale=None, v_scale=None), type=1), dict(cache=_cache(format=1, k_scale=None, v_scale=None), type=0),
                   # more pieces of work than 2^31
                   dict(batch=_batch(n_tokens=1 << 28, max_pages=1 << 20))):
        assert call(**change) == bad, change
    out = ctypes.c_int64(0)
    for args in ((0, 64), (8, 0), (8, 48), (8, 288)):
        assert lib.qtea_attention_workspace_bytes(*args, ctypes.byref(out)) == bad
    assert lib.qtea_attention_workspace_bytes(8, 64, None) == bad


def test_verification_refuses(lib):
    need = q.qtea_verify_workspace_bytes(2)

    def call(target=ADDR, draft=ADDR, type=2, vocab=100, ts=100, ds=100, tokens=ADDR, start=ADDR, ua=ADDR, us=ADDR, n_seq=2, rows=5, drafts=3,
             most=2, acc=ADDR, out=ADDR, ws=ADDR, nbytes=need):
        return lib.qtea_verify_draft(target, draft, type, vocab, ts, ds, tokens, start, ua, us, n_seq, rows, drafts, most, acc, out, ws, nbytes, None)

    bad = q.QTEA_ERR_INVALID_ARG
    for change in (dict(target=None), dict(start=None), dict(us=None), dict(acc=None), dict(out=None), dict(ws=None), dict(tokens=None), dict(ua=None),
                   dict(type=3), dict(type=-1), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(ts=99), dict(ds=99), dict(ts=1 << 40),
                   dict(n_seq=0), dict(rows=-1), dict(rows=1 << 31), dict(drafts=-1), dict(drafts=1 << 31), dict(most=-1), dict(most=1024),
                   dict(target=VP((1 << 20) + 2)), dict(ws=VP((1 << 20) + 8))):
        assert call(**change) == bad, change
    assert call(nbytes=need - 1) == q.QTEA_ERR_WORKSPACE
    out = ctypes.c_int64(0)
    assert lib.qtea_verify_workspace_bytes(0, ctypes.byref(out)) == bad
    assert lib.qtea_verify_workspace_bytes(3, None) == bad


def test_the_binding_refuses():
    z = lambda *s, dt=torch.uint8: torch.zeros(s, dtype=dt)  # noqa: E731
    with pytest.raises(ValueError):
        q.KvCache("e5m2", z(2, 1, 16, 64), z(2, 1, 16, 64))
    with pytest.raises(ValueError):
        q.KvCache("e4m3", z(2, 1, 16, 64), z(2, 1, 16, 64))  # no scales
    with pytest.raises(ValueError):
        q.KvCache("f16", z(2, 1, 16, 64, dt=torch.bfloat16), z(2, 1, 16, 64, dt=torch.bfloat16))
    with pytest.raises(ValueError):
        q.KvCache("e4m3", z(2, 1, 16, 64), z(2, 1, 16, 64), z(2, 1, 16, 3), z(2, 1, 16, 2))
    with pytest.raises(ValueError):  # host tensors
        q.KvCache("f16", z(2, 1, 16, 64, dt=torch.float16), z(2, 1, 16, 64, dt=torch.float16))
    i32, f32 = torch.int32, torch.float32
    with pytest.raises(ValueError):
        q.qtea_verify_draft(z(3, 9, dt=f32), z(2, 8, dt=f32), z(2, dt=i32), z(2, dt=i32), z(2, dt=f32), z(1, dt=f32), z(1, dt=i32), z(1, 3, dt=i32), z(64))
    with pytest.raises(ValueError):
        q.qtea_verify_draft(z(3, 9, dt=f32), z(2, 9, dt=f32), z(2, dt=torch.int64), z(2, dt=i32), z(2, dt=f32), z(1, dt=f32), z(1, dt=i32), z(1, 3, dt=i32), z(64))


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_oracle_blocks(fmt):
    """The chosen scale is the smallest without saturation, every value of the
    result an fp16 and a bf16 value, no other code nearer."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((400, 64)).astype(np.float32) * (2.0 ** rng.integers(-30, 20, (400, 1))).astype(np.float32)
    code, scale = sv.encode(x.astype(np.float64), fmt)
    got = sv.decode(code, scale, fmt)
    top, (low, high) = sv.LADDER[fmt][-1], sv.EXPONENTS[fmt]
    e = scale.astype(int) - 127
    amax = np.abs(x).reshape(400, 2, 32).max(-1)
    assert ((amax <= top * 2.0 ** e) | (e == high)).all() and ((amax > top * 2.0 ** (e - 1)) | (e == low)).all()
    t = torch.from_numpy(got)
    assert torch.equal(t.half().double(), t) and torch.equal(t.bfloat16().double(), t)
    ladder = np.concatenate([-sv.LADDER[fmt], sv.LADDER[fmt]])
    unit = np.repeat(2.0 ** e, 32, -1)
    nearest = np.abs(np.clip(x, -top * unit, top * unit)[..., None] - ladder * unit[..., None]).min(-1)
    np.testing.assert_array_equal(np.abs(np.clip(x, -top * unit, top * unit) - got), nearest)
    # NaN and infinities take their block with them
    x[0, 3], x[1, 40] = np.nan, -np.inf
    bad = np.isnan(sv.decode(*sv.encode(x.astype(np.float64), fmt), fmt))
    assert bad[0, :32].all() and bad[1, 32:].all() and bad.sum() == 64


def test_oracle_verification_by_hand():
    p, d = np.array([[0.5, 0.25, 0.25], [0.0, 0.0, 1.0]]), np.array([[0.25, 0.75, 0.0]])
    assert sv.verify(p, d, [1], [0.3], 0.9) == (1, 2)          # 0.3 < 1/3: kept, then the last row's token
    assert sv.verify(p, d, [1], [0.34], 0.4) == (0, 0)         # residual (0.25, 0, 0.25): the lower half
    assert sv.verify(p, d, [1], [0.34], 0.5) == (0, 2)
    assert sv.verify(p, None, [1], [0.25], 0.7) == (0, 2)      # deterministic draft: kept below 0.25 only
    assert sv.verify(p, None, [1], [0.2], 0.7) == (1, 2)
    assert sv.verify(np.zeros((2, 3)), d, [1], [0.5], 0.5) == (0, -1)
