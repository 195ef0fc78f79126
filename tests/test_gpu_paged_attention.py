"""qtea_paged_attention against the oracle in fp64, within the bound derived
in tests/serving_cases.py."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2609_00224_amd as q
from tests.serving_cases import TORCH, Paged, attention_reference, rounded

pytestmark = pytest.mark.gpu


def _types(fmt):
    return [fmt] if fmt in ("f16", "bf16") else ["f16", "bf16"]


def _run(p, Q, window=0, scale=None, ws=None, cache=None, meta=None):
    out = torch.full(Q.shape, 7.0, dtype=TORCH[p.qtype], device="cuda")
    q.qtea_paged_attention(cache or p.cache(), torch.from_numpy(Q).to(TORCH[p.qtype]).cuda(), *(meta or p.meta()), out,
                           q.new_attention_workspace(Q.shape[1], p.dim) if ws is None else ws, scale=scale, window=window)
    return out.double().cpu().numpy()


def _check(p, Q, got, window=0, scale=None):
    want, bound = attention_reference(p, Q, p.dim ** -0.5 if scale is None else scale, window)
    assert got.shape == want.shape and np.isfinite(got).all()
    worst = np.max(np.abs(got - want) - bound)
    assert worst <= 0, f"off by {np.abs(got - want).max():.3g}, {worst:.3g} over the bound"


def _case(seed, lens, heads, group, dim, page, fmt, qtype, sharp=1.0):
    rng = np.random.default_rng(seed)
    p = Paged(rng, lens, heads, dim, page, fmt)
    p.qtype = qtype
    return p, rounded(rng.standard_normal((p.rows, heads * group, dim)) * sharp, qtype)


LENGTHS = {
    "one token": [(1, 1)],
    "tile edges": [(15, 1), (16, 1), (17, 1), (31, 1), (32, 1), (33, 1), (127, 1), (128, 1), (129, 1), (255, 1), (257, 1)],
    "whole prompts": [(1, 1), (5, 5), (64, 64), (131, 131)],
    "drafts": [(700, 4), (33, 6), (6, 6), (1025, 1), (90, 3)],
    "chunks": [(400, 150), (1000, 33), (61, 60), (300, 1)],
    "empty ones": [(0, 0), (50, 0), (70, 2), (0, 0), (9, 1), (12, 0)],
    "long": [(9001, 2)],
}
HEADS = [(1, 1, 32), (8, 4, 128), (2, 5, 128), (1, 16, 64), (2, 8, 256), (3, 3, 96), (1, 40, 128), (2, 1, 160)]


@pytest.mark.parametrize("fmt,qtype", [(f, t) for f in ("f16", "bf16", "e4m3", "e2m1") for t in _types(f)])
@pytest.mark.parametrize("lengths", sorted(LENGTHS))
def test_lengths(lengths, fmt, qtype):
    p, Q = _case([1, len(lengths)], LENGTHS[lengths], 2, 4, 128, 16, fmt, qtype)
    _check(p, Q, _run(p, Q))


@pytest.mark.parametrize("fmt,qtype", [("f16", "f16"), ("bf16", "bf16"), ("e4m3", "f16"), ("e2m1", "bf16")])
@pytest.mark.parametrize("heads,group,dim", HEADS)
def test_heads_and_channels(heads, group, dim, fmt, qtype):
    for page, lens in ((16, [(300, 1), (75, 2)]), (64, [(200, 70), (40, 40)])):
        p, Q = _case([2, heads, group, dim], lens, heads, group, dim, page, fmt, qtype)
        _check(p, Q, _run(p, Q))


@pytest.mark.parametrize("fmt,qtype", [("f16", "f16"), ("e4m3", "bf16"), ("e2m1", "f16")])
@pytest.mark.parametrize("window", [1, 7, 16, 33, 128, 1000])
def test_windows(window, fmt, qtype):
    for group, lens in ((4, [(500, 1), (20, 20), (300, 3), (1, 1)]), (3, [(400, 200), (130, 130)])):
        p, Q = _case([3, window, group], lens, 2, group, 64, 32, fmt, qtype)
        _check(p, Q, _run(p, Q, window), window)


@pytest.mark.parametrize("new", [1, 5, 90])
def test_pages_left_behind_by_the_window_are_not_read(new):
    """Their table entries may be anything."""
    p, Q = _case([4, new], [(1000, new), (600, new)], 2, 4, 128, 16, "e4m3", "f16")
    window = 100
    meta = list(p.meta())
    for s, (c, n) in enumerate(p.lens):
        gone = (c - n + 1 - window) // 16  # whole pages below the first row's window
        meta[2][s, :gone] = torch.tensor([-1, 1 << 30], dtype=torch.int32).repeat(gone)[:gone]
    _check(p, Q, _run(p, Q, window, meta=meta), window)


@pytest.mark.parametrize("seqs", [1, 63, 64, 65, 200])
def test_many_sequences(seqs):
    rng = np.random.default_rng([5, seqs])
    lens = [(int(c), int(rng.integers(0, 3)) if c > 2 else 0) for c in rng.integers(0, 300, seqs)]
    lens[-1] = (77, 1)
    p, Q = _case([6, seqs], lens, 1, 4, 64, 16, "f16", "f16")
    _check(p, Q, _run(p, Q))


@pytest.mark.parametrize("sharp", [1e-3, 8.0, 60.0])
@pytest.mark.parametrize("new", [1, 40])
def test_flat_and_sharp_scores(new, sharp):
    """Weights all alike, and one that takes all (running maxima that move often)."""
    p, Q = _case([7, new], [(2000, new)], 1, 4, 128, 64, "f16", "f16", sharp)
    _check(p, Q, _run(p, Q))
    _check(p, Q, _run(p, Q, scale=0.5), scale=0.5)


@pytest.mark.parametrize("new", [1, 4, 70])
def test_negative_positions_become_zero(new):
    """More new rows than the sequence has positions: the first see nothing."""
    p, Q = _case([8, new], [(max(0, new - 3), new), (50, 1)], 2, 4, 128, 16, "f16", "f16")
    got = _run(p, Q)
    _check(p, Q, got)
    assert (got[:min(3, new)] == 0).all()


@pytest.mark.parametrize("fmt,qtype", [("f16", "f16"), ("bf16", "bf16"), ("e4m3", "f16"), ("e2m1", "f16")])
@pytest.mark.parametrize("new,window", [(1, 0), (6, 0), (6, 40), (100, 0), (100, 40)])
def test_what_a_row_does_not_see_does_not_reach_it(new, window, fmt, qtype):
    """NaN and infinities past a sequence's end, below its window and among
    the later tokens of its own chunk."""
    p, Q = _case([9, new, window], [(150, new)], 2, 4, 128, 64, fmt, qtype)
    cache = p.cache()
    want = _run(p, Q, window, cache=cache)
    pg, off = p.places(0, 0, 150)
    end = [(int(p.table[0, 2]), slice(150 % 64, 64))]
    low = [(int(pg[t]), int(off[t])) for t in range(max(0, 150 - new + 1 - window))] if window else []
    quant = cache.k_scale is not None
    for at_page, at_off in end + low:
        for pool in ((cache.k_scale, cache.v_scale) if quant else (cache.k, cache.v)):
            pool[at_page, :, at_off] = 255 if quant else float("nan")
    np.testing.assert_array_equal(_run(p, Q, window, cache=cache), want)
    if new == 1:
        return
    # the last token's V: only the last row may change (both of its kinds of values)
    for value in ((255,) if quant else (float("nan"), float("inf"), float("-inf"))):
        (cache.v_scale if quant else cache.v)[int(pg[149]), :, int(off[149])] = value
        got = _run(p, Q, window, cache=cache)
        np.testing.assert_array_equal(got[:-1], want[:-1])
        if quant or np.isnan(value):
            assert np.isnan(got[-1]).all()
        else:
            assert (got[-1] == value).all()
    # both infinities among what the last row sees; the row before sees one
    if not quant:
        cache.v[int(pg[148]), :, int(off[148])] = float("inf")
        got = _run(p, Q, window, cache=cache)
        np.testing.assert_array_equal(got[:-2], want[:-2])
        assert (got[-2] == np.inf).all() and np.isnan(got[-1]).all()
        cache.k[int(pg[149]), :, int(off[149])] = float("nan")
        got = _run(p, Q, window, cache=cache)
        np.testing.assert_array_equal(got[:-2], want[:-2])
        assert (got[-2] == np.inf).all() and np.isnan(got[-1]).all()


@pytest.mark.parametrize("new", [1, 80])
def test_a_bad_page_or_length_gives_nan(new):
    p, Q = _case([10, new], [(100, new), (100, new), (100, new)], 2, 4, 64, 16, "f16", "f16")
    meta = list(p.meta())
    clean = _run(p, Q, meta=meta)
    meta[2][0, 1] = p.pages
    meta[1][2] = 16 * p.table.shape[1] + 1
    got = _run(p, Q, meta=meta)
    assert np.isnan(got[:new]).all() and np.isnan(got[2 * new:]).all()
    np.testing.assert_array_equal(got[new:2 * new], clean[new:2 * new])


def test_strided_rows_and_rows_of_no_sequence():
    p, Q = _case(11, [(90, 2), (300, 1)], 2, 4, 128, 16, "e4m3", "f16")
    wide = torch.full((p.rows + 3, 24, 128), 3.0, dtype=torch.float16, device="cuda")
    wide[:p.rows, 8:16] = torch.from_numpy(Q)
    res = torch.full((p.rows + 3, 16, 128), 5.0, dtype=torch.float16, device="cuda")
    q.qtea_paged_attention(p.cache(), wide[:, 8:16], *p.meta(), res[:, :8], q.new_attention_workspace(8, 128))
    _check(p, Q, res[:p.rows, :8].double().cpu().numpy())
    assert (res[p.rows:] == 5.0).all() and (res[:, 8:] == 5.0).all()


def test_a_workspace_serves_any_sequence_of_calls_the_same_way():
    """Deterministic, and clean after every call: other shapes in between."""
    ws = q.new_attention_workspace(8, 128)
    cases = [_case([12, i], lens, 2, 4, 128, 16, "e4m3", "f16")
             for i, lens in enumerate(([(5000, 1)], [(300, 200)], [(40, 4)] * 9, [(3000, 3), (2, 1)]))]
    first = [_run(p, Q, ws=ws) for p, Q in cases]
    for _ in range(3):
        for (p, Q), want in zip(cases, first):
            np.testing.assert_array_equal(_run(p, Q, ws=ws), want)
    for (p, Q), got in zip(cases, first):
        _check(p, Q, got)


@pytest.mark.parametrize("new", [1, 50])
def test_in_a_graph_as_the_lengths_grow(new):
    p, Q = _case([13, new], [(400, new), (150, new)], 2, 4, 128, 16, "e2m1", "f16")
    cache, meta = p.cache(), p.meta()
    qd, out, ws = torch.from_numpy(Q).half().cuda(), torch.empty(Q.shape, dtype=torch.float16, device="cuda"), q.new_attention_workspace(8, 128)
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        q.qtea_paged_attention(cache, qd, *meta, out, ws)
    full = p.k, p.v
    for c in (400, 230, 399):
        lens = [c, c // 4 + new]
        meta[1].copy_(torch.tensor(lens))
        g.replay()
        torch.cuda.synchronize()
        eager = torch.empty_like(out)
        q.qtea_paged_attention(cache, qd, *meta, eager, ws)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        p.lens = [(n, new) for n in lens]
        p.k, p.v = ([x[:n] for x, n in zip(vals, lens)] for vals in full)
        _check(p, Q, out.double().cpu().numpy())
