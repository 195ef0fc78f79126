"""The serving operators' binding and entry points at the edges of their
arguments, as far as no device is needed."""
from __future__ import annotations

import contextlib
import ctypes
import os
import subprocess
import sys
import types

import pytest
import torch

import paper_2609_00224_amd as q


class Calls:
    """Stands for the library: records the calls it gets."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        if not name.startswith("qtea_"):
            raise AttributeError(name)
        return lambda *args: self.made.append((name, args)) or q.QTEA_OK


@pytest.fixture
def calls(monkeypatch):
    got = Calls()
    monkeypatch.setattr(q, "load", lambda: got)
    return got


def _cache(device=-1, heads=2, dim=64):
    return types.SimpleNamespace(device_index=device, n_heads=heads, head_dim=dim, desc=q.QteaKvCache())


def _attend(window=0, stream=types.SimpleNamespace(cuda_stream=0), rows=3, heads=4, dim=64, cache=None):
    t = torch.zeros((rows, heads, dim), dtype=torch.float16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q.qtea_paged_attention(cache or _cache(), t, i32(3), i32(2), i32(2, 5), t, torch.zeros(64, dtype=torch.uint8), window=window, stream=stream)


@pytest.mark.parametrize("window,passed", [(0, 0), (1, 1), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1), (2 ** 32, 2 ** 31 - 1), (2 ** 32 + 5, 2 ** 31 - 1),
                                           (2 ** 63 - 1, 2 ** 31 - 1), (10 ** 30, 2 ** 31 - 1)])
def test_a_window_past_the_types_range_is_the_largest(calls, window, passed):
    _attend(window)
    (name, args), = calls.made
    assert name == "qtea_paged_attention" and args[9] == passed


@pytest.mark.parametrize("window", [-1, -2 ** 31, 5 - 2 ** 32])
def test_a_negative_window_stays_negative(calls, window):
    """The entry point refuses it."""
    _attend(window)
    (_, args), = calls.made
    assert args[9] == -1


@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
@pytest.mark.parametrize("off", [1, 4, 8])
def test_scale_pools_are_aligned(which, off):
    """They are read up to 16 bytes at a time."""
    addr = ctypes.c_void_p(1 << 20)  # never read: every call is refused
    f = dict(k=1 << 20, v=1 << 20, k_scale=1 << 20, v_scale=1 << 20, n_pages=4, format=2, n_heads=2, head_dim=64, page_size=16)
    cache = q.QteaKvCache(**{**f, which: (1 << 20) + off})
    batch = q.QteaKvBatch(q_start=1 << 20, kv_len=1 << 20, page_table=1 << 20, n_tokens=0, n_seq=2, max_pages=5)
    lib = q.load()
    for name in ("qtea_kv_append", "qtea_kv_read"):
        assert getattr(lib, name)(cache, batch, addr, addr, 2, 128, 128, None) == q.QTEA_ERR_INVALID_ARG
    assert lib.qtea_paged_attention(cache, batch, addr, addr, 0, 8, 512, 512, 0.1, 0, addr, 1 << 40, None) == q.QTEA_ERR_INVALID_ARG


class Devices:
    """Stands for torch.cuda with two devices, of which 0 is the current one."""

    def __init__(self, monkeypatch):
        self.current = 0
        monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: self.current)
        monkeypatch.setattr(torch.cuda, "device", self.guard)

    @contextlib.contextmanager
    def guard(self, device):
        before, self.current = self.current, device
        yield
        self.current = before


@pytest.mark.parametrize("current", [0, -1])  # (host tensors' device is -1)
def test_a_call_is_made_on_its_tensors_device(monkeypatch, current):
    devices, at = Devices(monkeypatch), []
    devices.current = current

    class On(Calls):
        def __getattr__(self, name):
            at.append(devices.current)
            return lambda *args: at.append(devices.current) or q.QTEA_OK

    monkeypatch.setattr(q, "load", On)
    stream = types.SimpleNamespace(cuda_stream=0)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    _attend(stream=stream)
    t = torch.zeros((3, 2, 64))
    q.qtea_kv_append(_cache(), t, t, i32(3), i32(2), i32(2, 5), stream=stream)
    q.qtea_kv_read(_cache(), i32(3), i32(2), i32(2, 5), t, t, stream=stream)
    assert at[1::2] == [-1] * 3 and devices.current == current


def test_the_package_and_its_host_entry_points_do_without_torch():
    """Torch is imported where tensors are, the serving operators' binding with them."""
    code = ("import sys; sys.modules['torch'] = None\n"
            "import paper_2609_00224_amd as q\n"
            "assert q.qtea_abi_version() == q.QTEA_ABI_VERSION and q.qtea_packed_bytes(64, 256, 3) > 0\n"
            "assert 'KvCache' in dir(q) and q.QteaKvCache and q.KV_FORMATS\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", code], cwd=root, check=True, timeout=120)


@pytest.mark.parametrize("scale,fits", [(2.3e38, True), (2.4e38, False), (3.0e38, False), (1e-45, True)])
def test_a_softmax_scale_whose_product_overflows_is_refused(scale, fits):
    """It would make every score infinite or NaN."""
    addr = ctypes.c_void_p(1 << 20)  # never read: refused, or no tokens
    cache = q.QteaKvCache(k=1 << 20, v=1 << 20, n_pages=4, format=0, n_heads=2, head_dim=64, page_size=16)
    batch = q.QteaKvBatch(q_start=1 << 20, kv_len=1 << 20, page_table=1 << 20, n_tokens=0, n_seq=2, max_pages=5)
    rc = q.load().qtea_paged_attention(cache, batch, addr, addr, 0, 8, 512, 512, scale, 0, addr, 1 << 40, None)
    assert (rc != q.QTEA_ERR_INVALID_ARG) == fits


@pytest.mark.parametrize("page", [16, 4096])
def test_the_largest_page_table(page):
    """Positions and what the kernels add to them are 32-bit numbers."""
    addr = ctypes.c_void_p(1 << 20)  # never read: refused, or no tokens
    cache = q.QteaKvCache(k=1 << 20, v=1 << 20, n_pages=4, format=0, n_heads=2, head_dim=64, page_size=page)
    lib = q.load()
    for most, fits in (((2 ** 31 - 1 - 8192) // page, True), ((2 ** 31 - 1) // page, False)):
        batch = q.QteaKvBatch(q_start=1 << 20, kv_len=1 << 20, page_table=1 << 20, n_tokens=0, n_seq=2, max_pages=most)
        for name in ("qtea_kv_append", "qtea_kv_read"):
            assert (getattr(lib, name)(cache, batch, addr, addr, 2, 128, 128, None) == q.QTEA_OK) == fits
        rc = lib.qtea_paged_attention(cache, batch, addr, addr, 0, 8, 512, 512, 0.1, 0, addr, 1 << 40, None)
        assert (rc != q.QTEA_ERR_INVALID_ARG) == fits
