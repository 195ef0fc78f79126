"""Serving operators at the edges of what their arguments may be."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.serving as sv
import paper_2609_00224_amd as q
from tests.serving_cases import TORCH, Paged, attention_reference, pack, rounded
from tests.test_gpu_verify_draft import _inputs, _run, _want

pytestmark = pytest.mark.gpu


def test_one_verification_workspace_serves_batches_of_any_size():
    """Made for the largest batch, then used for smaller and larger ones in turn."""
    rng = np.random.default_rng(20)
    ws = q.new_verify_workspace(48)
    for seqs, vocab in ((48, 65), (1, 20000), (7, 300), (48, 65), (2, 5003), (48, 65)):
        x = _inputs(rng, [int(k) for k in rng.integers(1, 4, seqs)], vocab, "f32")
        got, want = _run(x, 3, ws=ws), _want(x, 3)
        np.testing.assert_array_equal(got[0], want[0])
        np.testing.assert_array_equal(got[1], want[1])


@pytest.mark.parametrize("deterministic", [False, True])
@pytest.mark.parametrize("ahead", [1, 4])
def test_the_first_sequences_drafts_come_first_wherever_its_rows_start(ahead, deterministic):
    """Target rows of no sequence before the first: the drafts do not move."""
    rng = np.random.default_rng([21, ahead])
    x = _inputs(rng, [2, 0, 3, 1], 500, "f32")
    if deterministic:
        del x["draft"]
    want = _want(x, 3)
    x["target"] = torch.cat((torch.rand((ahead, 500)), x["target"]))
    x["q_start"] = x["q_start"] + ahead
    got = _run(x, 3)
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])


@pytest.mark.parametrize("with_draft", [False, True])
def test_a_verification_without_any_rows(with_draft):
    z = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    acc, out = torch.full((3,), 99, dtype=torch.int32, device="cuda"), torch.full((3, 3), 99, dtype=torch.int32, device="cuda")
    rows = z(0, 50, dt=torch.float32)
    q.qtea_verify_draft(rows, rows if with_draft else None, z(0), z(4), z(0, dt=torch.float32), z(3, dt=torch.float32), acc, out, q.new_verify_workspace(3))
    assert (acc == 0).all() and (out == -1).all()


def _large_scale_case(new, window, fmt, qtype, byte, seed):
    """One sequence of 150 positions, the last `new` of them new."""
    rng = np.random.default_rng([22, new, window, byte, seed])
    p = Paged(rng, [(150, new)], 2, 64, 64, fmt)
    p.qtype = qtype
    Q = rounded(rng.standard_normal((new, 4, 64)), qtype)
    return rng, p, Q


def _attend(p, Q, window, cache):
    out = torch.full(Q.shape, 7.0, dtype=TORCH[p.qtype], device="cuda")
    q.qtea_paged_attention(cache, torch.from_numpy(Q).to(TORCH[p.qtype]).cuda(), *p.meta(), out, q.new_attention_workspace(Q.shape[1], p.dim), window=window)
    return out.double().cpu().numpy()


def _poison(cache, fmt, page, off, byte, codes):
    """Token's V: scale bytes and codes ([32] per block, the same for all)."""
    cache.v_scale[page, :, off] = byte
    row = np.concatenate([codes] * 2)
    if fmt == "e2m1":
        row = row[0::2] | (row[1::2] << 4)
    cache.v[page, :, off] = torch.from_numpy(row.astype(np.uint8)).cuda()


# Codes of a block: the largest, small and zero ones side by side.
CODES = {"e4m3": np.array([0x7e, 0x00, 0x08, 0xfe] * 8, np.uint8), "e2m1": np.array([7, 0, 1, 15, 1, 7, 0, 9] * 4, np.uint8)}


def _check_seen(new, qtype, fmt, byte):
    """The newest token's V, which only the last row sees: a channel whose
    value rounds to an infinity of the type is that infinity, the others are
    finite, and no other row changes."""
    rng, p, Q = _large_scale_case(new, 0, fmt, qtype, byte, 1)
    cache = p.cache()
    want = _attend(p, Q, 0, cache)
    pg, off = p.places(0, 0, 150)
    _poison(cache, fmt, int(pg[149]), int(off[149]), byte, CODES[fmt])
    got = _attend(p, Q, 0, cache)
    np.testing.assert_array_equal(got[:-1], want[:-1])
    value = sv.decode(np.concatenate([CODES[fmt]] * 2), np.array([byte] * 2, np.uint8), fmt)
    as_type = torch.from_numpy(value).to(TORCH[qtype]).double().numpy()
    inf = np.isinf(as_type)
    np.testing.assert_array_equal(got[-1][:, inf], np.broadcast_to(as_type[inf], (4, int(inf.sum()))))
    assert not np.isnan(got[-1]).any()
    # a share of a finite value and of the others' values
    assert (np.abs(got[-1][:, ~inf]) <= 1.01 * (np.abs(as_type[~inf]) + np.abs(p.v[0]).max())).all()


@pytest.mark.parametrize("byte", [135, 141, 200, 247, 253])
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("qtype", ["f16", "bf16"])
def test_seen_values_past_the_types_range_reach_their_rows_and_channels_many_rows(qtype, fmt, byte):
    _check_seen(100, qtype, fmt, byte)


@pytest.mark.parametrize("byte", [134, 135, 140, 141, 200, 246, 247, 252, 253, 254])
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("qtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,window", [(1, 0), (6, 40), (100, 40)])
def test_unseen_values_past_the_types_range_do_not_reach_a_row(new, window, qtype, fmt, byte):
    """Past a sequence's end and below its window: any code and any scale."""
    rng, p, Q = _large_scale_case(new, window, fmt, qtype, byte, 0)
    cache = p.cache()
    want = _attend(p, Q, window, cache)
    pg, off = p.places(0, 0, 150)
    unseen = [(int(p.table[0, 2]), o) for o in range(150 % 64, 64)]
    unseen += [(int(pg[t]), int(off[t])) for t in range(max(0, 150 - new + 1 - window))] if window else []
    for page, o in unseen:
        _poison(cache, fmt, page, o, byte, rng.permutation(CODES[fmt]))
    np.testing.assert_array_equal(_attend(p, Q, window, cache), want)


@pytest.mark.parametrize("byte", [135, 141, 200, 247, 253])
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("qtype", ["f16", "bf16"])
@pytest.mark.parametrize("new", [2, 20])
def test_seen_values_past_the_types_range_reach_their_rows_and_channels_few_rows(new, qtype, fmt, byte):
    _check_seen(new, qtype, fmt, byte)


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("qtype", ["f16", "bf16"])
@pytest.mark.parametrize("new", [2, 100])
def test_every_scale_and_code_of_a_token_that_one_row_sees(new, qtype, fmt):
    """As above, all of a format's codes over 8 blocks, scales from where the
    largest of them is finite to where every one but zero is not."""
    rng = np.random.default_rng([26, new])
    p = Paged(rng, [(90, new)], 1, 256, 32, fmt)
    p.qtype = qtype
    Q = rounded(rng.standard_normal((new, 1, 256)), qtype)
    cache = p.cache()
    want = _attend(p, Q, 0, cache)
    pg, off = p.places(0, 0, 90)
    codes = np.arange(256) if fmt == "e4m3" else np.tile(np.arange(16), 16)
    codes = rng.permutation(codes).astype(np.uint8)
    at = int(pg[89]), 0, int(off[89])
    cache.v[at] = torch.from_numpy(pack(codes, fmt)).cuda()
    for byte in range(132, 166) if qtype == "f16" else range(244, 256):
        cache.v_scale[at] = byte
        got = _attend(p, Q, 0, cache)
        np.testing.assert_array_equal(got[:-1], want[:-1])
        value = sv.decode(codes, np.full(8, byte, np.uint8), fmt)
        as_type = torch.from_numpy(value).to(TORCH[qtype]).double().numpy()
        wild = ~np.isfinite(as_type)
        np.testing.assert_array_equal(got[-1][0, wild], as_type[wild])
        assert (np.abs(got[-1][0, ~wild]) <= 1.01 * (np.abs(as_type[~wild]) + np.abs(p.v[0]).max())).all()


@pytest.mark.parametrize("new", [5, 90])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 4, 2 ** 30])
def test_the_largest_windows_with_more_rows_than_positions(window, new):
    rng = np.random.default_rng([23, new])
    p = Paged(rng, [(new - 3, new), (50, 1), (1, new)], 2, 64, 16, "f16")
    p.qtype = "f16"
    Q = rounded(rng.standard_normal((p.rows, 8, 64)), "f16")
    got = _attend(p, Q, window, p.cache())
    want, bound = attention_reference(p, Q, 0.125)
    assert (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_a_scale_byte_of_zero_is_two_to_the_minus_127(fmt):
    rng = np.random.default_rng(24)
    p = Paged(rng, [(20, 20)], 2, 64, 16, fmt)
    cache = p.cache()
    for t in (cache.k_scale, cache.v_scale):
        t[int(p.table[0, 0])] = 0
    k, v = (torch.empty((20, 2, 64), device="cuda") for _ in range(2))
    q.qtea_kv_read(cache, *p.meta(), k, v)
    for got, vals, scale in ((k, p.k, p.pool["k"][1]), (v, p.v, p.pool["v"][1])):
        old = np.repeat(scale.numpy()[p.table[0, 0]].transpose(1, 0, 2).astype(np.float64), 32, -1)
        want = vals[0].copy()
        want[:16] *= 2.0 ** -old
        assert torch.equal(got.cpu().double(), torch.from_numpy(want))


@pytest.mark.parametrize("new", [1, 100])
@pytest.mark.parametrize("fmt,code", [("e4m3", 0x7e), ("e4m3", 0xc8), ("e2m1", 7), ("e2m1", 12)])
def test_a_scale_byte_of_zero_in_attention(fmt, code, new):
    """One value everywhere (a normal bf16 one): every average is that value."""
    rng = np.random.default_rng(25)
    p = Paged(rng, [(120, new)], 2, 64, 16, fmt)
    p.qtype = "bf16"
    cache = p.cache()
    cache.v.fill_(code if fmt == "e4m3" else code * 17)
    cache.v_scale.zero_()
    value = sv.decode(np.full(32, code, np.uint8), np.zeros(1, np.uint8), fmt)[0]
    got = _attend(p, rounded(rng.standard_normal((new, 8, 64)), "bf16"), 0, cache)
    assert (np.abs(got / value - 1) <= 1.02 * 2.0 ** -7).all()


def test_one_token_of_any_stride():
    """Of a single token no stride is used: a view with an odd one."""
    rng = np.random.default_rng(25)
    p = Paged(rng, [(40, 1)], 2, 64, 16, "f16")
    p.qtype = "f16"
    row = lambda x: torch.as_strided(x.reshape(-1), (1, x.shape[1], 64), (1001, 64, 1))  # noqa: E731
    Q = rounded(rng.standard_normal((1, 8, 64)), "f16")
    cache, meta = p.cache(), p.meta()
    k, v = (torch.randn((1, 2, 64), device="cuda").half() for _ in range(2))
    q.qtea_kv_append(cache, row(k), row(v), *meta)
    gk, gv = torch.zeros_like(k), torch.zeros_like(v)
    q.qtea_kv_read(cache, *meta, row(gk), row(gv))
    assert torch.equal(gk, k) and torch.equal(gv, v)
    p.k[0][39], p.v[0][39] = k[0].double().cpu().numpy(), v[0].double().cpu().numpy()
    out = torch.zeros((1, 8, 64), dtype=torch.float16, device="cuda")
    q.qtea_paged_attention(cache, row(torch.from_numpy(Q).half().cuda()), *meta, row(out), q.new_attention_workspace(8, 64))
    want, bound = attention_reference(p, Q, 0.125)
    assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()
