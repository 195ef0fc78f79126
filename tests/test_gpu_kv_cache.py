"""qtea_kv_append and qtea_kv_read against the oracle's format: codes, scales
and values bit for bit."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.serving as sv
import paper_2609_00224_amd as q
from tests.serving_cases import TORCH, Paged, pack, rounded

pytestmark = pytest.mark.gpu

CASES = [  # lengths (cached, new), heads, dim, page
    ([(1, 1)], 1, 32, 16),
    ([(1, 1), (0, 0), (33, 1), (200, 0), (64, 64)], 8, 128, 16),
    ([(100, 7), (131, 131), (17, 16)], 5, 96, 32),
    ([(77, 30)], 3, 256, 64),
    ([(40, 9), (300, 1)], 2, 64, 256),
    ([(20 + s, 1 + s % 3) for s in range(70)], 1, 64, 16),  # more sequences than a wave has lanes
    ([(30, 5)], 7, 160, 16),
]


def _news(rng, p, src):
    """New keys and values of magnitudes from 2^-20 to 2^17 by block, with
    zeros and exact ties among them."""
    shape = (p.rows, p.heads, p.dim // 32, 32)
    got = []
    for _ in range(2):
        mag = 2.0 ** rng.integers(-20, 18 if src != "f16" else 15, shape[:3])
        x = rng.standard_normal(shape) * mag[..., None]
        x[rng.random(shape[:3]) < 0.1] = 0.0
        tie = rng.random(shape[:3]) < 0.2  # whole and half steps of a coarse grid
        x = np.where(tie[..., None], np.round(rng.uniform(-28, 28, shape)) * 0.25 * mag[..., None], x)
        got.append(rounded(np.clip(x, -65504, 65504) if src == "f16" else x, src).reshape(p.rows, p.heads, p.dim))
    return got


def _expected(p, fmt, news):
    """The pools after the append, as the cache's tensors."""
    want = {}
    for w, x in zip(("k", "v"), news):
        codes, scale = (None if t is None else t.clone() for t in p.pool[w])
        for s, (c, n) in enumerate(p.lens):
            if n == 0:
                continue
            pg, off = p.places(s, c - n, c)
            part = x[p.q_start[s]:p.q_start[s + 1]]
            if fmt in ("f16", "bf16"):
                codes[pg, :, off] = torch.from_numpy(part).float().to(TORCH[fmt])
            else:
                cd, sc = sv.encode(part, fmt)
                codes[pg, :, off], scale[pg, :, off] = torch.from_numpy(pack(cd, fmt)), torch.from_numpy(sc)
        want[w] = (codes, scale)
    return want


def _same(a, b):
    """Equal bits, but for the sign of a zero."""
    if a.dtype != torch.uint8:
        return torch.equal(a.cpu().view(torch.int16), b.view(torch.int16)) or torch.equal(a.cpu(), b)
    return torch.equal(a.cpu(), b)


@pytest.mark.parametrize("src", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("fmt", ["f16", "bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_append_writes_the_oracles_codes_and_nothing_else(case, fmt, src):
    rng = np.random.default_rng([case, len(fmt), len(src)])
    p = Paged(rng, *CASES[case], fmt)
    news = _news(rng, p, src)
    # columns of one wider tensor: strided rows
    wide = torch.zeros((p.rows, 2 * p.heads + 1, p.dim), dtype=TORCH[src], device="cuda")
    k, v = wide[:, :p.heads], wide[:, p.heads:2 * p.heads]
    k.copy_(torch.from_numpy(news[0]))
    v.copy_(torch.from_numpy(news[1]))
    cache = p.cache()
    q.qtea_kv_append(cache, k, v, *p.meta())
    want = _expected(p, fmt, news)
    assert _same(cache.k, want["k"][0]) and _same(cache.v, want["v"][0])
    if cache.k_scale is not None:
        assert torch.equal(cache.k_scale.cpu(), want["k"][1]) and torch.equal(cache.v_scale.cpu(), want["v"][1])


@pytest.mark.parametrize("to", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("fmt", ["f16", "bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_read_gives_the_cached_values(case, fmt, to):
    rng = np.random.default_rng([7, case, len(fmt)])
    p = Paged(rng, *CASES[case], fmt)
    wide = torch.full((p.rows + 2, 2 * p.heads, p.dim), 9.0, dtype=TORCH[to], device="cuda")
    k, v = wide[:, :p.heads], wide[:, p.heads:]
    q.qtea_kv_read(p.cache(), *p.meta(), k, v)
    for got, vals in ((k, p.k), (v, p.v)):
        for s, (c, n) in enumerate(p.lens):
            want = torch.from_numpy(vals[s][c - n:c]).to(TORCH[to])
            assert torch.equal(got[p.q_start[s]:p.q_start[s + 1]].cpu(), want)
        assert (got[p.rows:] == 9.0).all()  # rows of no sequence stay as they are


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_blocks_that_are_not_finite_read_as_nan(fmt):
    rng = np.random.default_rng(1)
    p = Paged(rng, [(50, 4)], 2, 64, 16, fmt)
    x = torch.randn((4, 2, 64), device="cuda")
    x[0, 0, 3], x[1, 1, 40], x[2, 0, 63] = float("nan"), float("inf"), float("-inf")
    cache, meta = p.cache(), p.meta()
    q.qtea_kv_append(cache, x, x, *meta)
    k, v = torch.empty_like(x), torch.empty_like(x)
    q.qtea_kv_read(cache, *meta, k, v)
    nan = torch.zeros((4, 2, 2), dtype=torch.bool)
    nan[0, 0, 0] = nan[1, 1, 1] = nan[2, 0, 1] = True
    for got in (k, v):
        assert torch.equal(got.isnan().cpu(), nan.repeat_interleave(32, -1))


def test_rows_without_a_place_are_not_written_and_read_as_stated():
    """More new rows than positions, a page outside the pool, a length outside the table."""
    rng = np.random.default_rng(2)
    p = Paged(rng, [(3, 5), (40, 4), (20, 2), (18, 3)], 2, 32, 16, "f16")
    p.table[1, 2] = p.pages  # the page of positions 32..47
    p.kv_len[2] = 16 * p.table.shape[1] + 1
    p.table[3, 1] = -5       # the page of positions 16..17
    cache, meta = p.cache(), p.meta()
    before = cache.k.clone()
    x = torch.randn((p.rows, 2, 32), device="cuda").half()
    q.qtea_kv_append(cache, x, x, *meta)
    changed = (cache.k != before).any(-1).any(1).cpu()  # [page][offset]
    want = torch.zeros_like(changed)
    want[p.table[0, 0], 0:3] = True
    want[p.table[3, 0], 15] = True
    assert torch.equal(changed, want)
    assert torch.equal(cache.k[p.table[0, 0], :, 0:3].transpose(0, 1), x[2:5])
    k, v = torch.full_like(x, 5.0), torch.full_like(x, 5.0)
    q.qtea_kv_read(cache, *meta, k, v)
    assert (k[:2] == 0).all() and torch.equal(k[2:5], x[2:5])
    assert k[5:11].isnan().all() and torch.equal(k[11], x[11]) and k[12:].isnan().all()


def test_on_a_stream_of_its_own_and_in_a_graph():
    rng = np.random.default_rng(3)
    p = Paged(rng, [(50, 3), (9, 9)], 4, 128, 16, "e4m3")
    cache, meta = p.cache(), p.meta()
    x = torch.zeros((p.rows, 4, 128), device="cuda")
    k, v = torch.empty_like(x), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q.qtea_kv_append(cache, x, x, *meta, stream=side)
    q.qtea_kv_read(cache, *meta, k, v, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert (k == 0).all()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        q.qtea_kv_append(cache, x, x, *meta)
        q.qtea_kv_read(cache, *meta, k, v)
    for i in range(4):
        x.copy_(torch.randn(x.shape, device="cuda") * 2.0 ** i)
        g.replay()
        torch.cuda.synchronize()
        code, scale = sv.encode(x.cpu().double().numpy(), "e4m3")
        want = torch.from_numpy(sv.decode(code, scale, "e4m3")).float()
        assert torch.equal(k.cpu(), want) and torch.equal(v.cpu(), want)


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes: the last page's rows."""
    heads, page, dim = 8, 4096, 128
    pages = (1 << 32) // (heads * page * dim) + 2
    cache = q.KvCache("e4m3", *(torch.zeros((pages, heads, page, dim), dtype=torch.uint8, device="cuda") for _ in range(2)),
                      *(torch.zeros((pages, heads, page, dim // 32), dtype=torch.uint8, device="cuda") for _ in range(2)))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    meta = i32([0, 2]), i32([page + 1]), i32([[0, pages - 1]])
    x = torch.ones((2, heads, dim), device="cuda")
    q.qtea_kv_append(cache, x, 2 * x, *meta)
    k, v = torch.empty_like(x), torch.empty_like(x)
    q.qtea_kv_read(cache, *meta, k, v)
    assert torch.equal(k, x) and torch.equal(v, 2 * x)
    assert int((cache.k[pages - 1] != 0).sum()) == heads * dim and int((cache.k[0] != 0).sum()) == heads * dim
    out = torch.empty((2, heads, dim), dtype=torch.float16, device="cuda")
    q.qtea_paged_attention(cache, torch.zeros_like(out), *meta, out, q.new_attention_workspace(heads, dim))
    # position p sees p zero rows of V and the rows of 2
    assert torch.allclose(out[0].float(), torch.full_like(x[0], 2 / page), rtol=2 ** -10)
    assert torch.allclose(out[1].float(), torch.full_like(x[0], 4 / (page + 1)), rtol=2 ** -10)
