"""The layer operators where their ranges end: small results, alignments, sizes
past 2^29, paths that only large or odd operands take."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.layer as ol
import paper_2609_00224_amd as q
from tests.layer_cases import TORCH, U, check, room, rounded

pytestmark = pytest.mark.gpu


# -- the gated activation -----------------------------------------------------------
def _gate_error(gate, want, out):
    """What fp32 may be off before the last rounding: an exp2 and a reciprocal of an
    ulp (two half ulps) each, the sum and three products half an ulp each.  Results
    that are not fp32 may carry the exponent's rounding too: t = -g log2(e) is off by
    half an ulp and by the constant's 2^-26, 1.2 |t| U, which moves exp(-g) by that times
    ln 2, and the result by no more of itself."""
    return U * np.abs(want) * (8 + (0 if out == "f32" else 1.25 * np.abs(gate)))


@pytest.mark.parametrize("x,out", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("bf16", "e4m3")])
@pytest.mark.parametrize("shift", [0, 1])
def test_gate_where_the_factor_leaves_32_bits(x, out, shift):
    """Gates of -75 to -260 times values up to the type's largest: the factor is
    below 2^-126 from -87.3 on, the result a normal number far beyond that."""
    rng = np.random.default_rng([len(x), len(out), shift])
    rows, dim = 7, 992
    gate = rounded(-rng.uniform(75, 260, (rows, dim)), x)
    up = rounded(rng.choice([-1, 1], (rows, dim)) * rng.uniform(1, 1.9, (rows, dim)) * 2.0 ** rng.integers(-10, 128, (rows, dim)), x)
    gate[:, 0::32], up[:, 0::32] = rounded(np.float64(-88), x), 1000
    wide = torch.zeros((rows, 2 * dim + shift), dtype=TORCH[x], device="cuda")
    wide[:, shift:] = torch.from_numpy(np.concatenate((gate, up), 1)).to(TORCH[x])
    got, scale = room((rows, dim), out)
    q.qtea_silu_mul(wide[:, shift:shift + dim], wide[:, shift + dim:], got, out_scale=scale)
    want = ol.silu_mul(gate, up)
    assert (np.abs(want) >= 2.0 ** -126).mean() > 0.2
    # (the last product in 32 bits may be rounded to its smallest step)
    check(got, scale, want, out, _gate_error(gate, want, out) + 2.0 ** -150)


def test_gate_far_below_and_not_finite():
    """Whatever a gate below -512 meets: 0 times finite values, the formula's
    infinity or NaN times the others."""
    inf, nan = float("inf"), float("nan")
    g = torch.tensor([[-513.0, -1e4, -3e38, -100.0, -1e4, -3e38, -100.0, -3e38, -inf, -inf, -600.0, nan, -90.0, -90.0, -81.0, -81.0]], device="cuda")
    u = torch.tensor([[3e38, -3e38, 3e38, inf, -inf, inf, nan, nan, 0.0, 1.0, 0.0, 1e30, 0.0, -0.0, inf, -1.0]], device="cuda")
    out = torch.empty_like(g)
    q.qtea_silu_mul(g, u, out)
    got = out[0].tolist()
    assert got[:3] == [0, 0, 0] and got[3] == -inf and got[4] == inf and got[5] == -inf and got[10] == 0 and got[12] == got[13] == 0 and got[14] == -inf
    assert out[0, [6, 7, 8, 9, 11]].isnan().all()
    assert abs(got[15] - 81 * np.exp(-81.0)) <= 8 * U * 81 * np.exp(-81.0)


@pytest.mark.parametrize("out", ["f16", "bf16", "f32", "e4m3"])
@pytest.mark.parametrize("x", ["f16", "bf16", "f32"])
def test_gate_has_the_same_bits_at_any_alignment(x, out):
    """Aligned rows, shifted inputs and a shifted output take different kernels."""
    rng = np.random.default_rng([len(x), len(out)])
    rows, dim = 40, 4096
    both = torch.from_numpy(rng.standard_normal((rows, 2 * dim)) * rng.choice([1, 10, 40], (rows, 2 * dim))).to(TORCH[x]).cuda()
    want, want_scale = room((rows, dim), out)
    q.qtea_silu_mul(both[:, :dim], both[:, dim:], want, out_scale=want_scale)
    wide = torch.zeros((rows, 2 * dim + 1), dtype=TORCH[x], device="cuda")
    wide[:, 1:] = both
    got, scale = room((rows, dim), out)
    q.qtea_silu_mul(wide[:, 1:1 + dim], wide[:, 1 + dim:], got, out_scale=scale)
    assert torch.equal(got, want) and (scale is None or torch.equal(scale, want_scale))
    if out != "e4m3":
        got = torch.zeros((rows, dim + 1), dtype=TORCH[out], device="cuda")[:, 1:]
        q.qtea_silu_mul(both[:, :dim], both[:, dim:], got)
        assert torch.equal(got, want)


@pytest.mark.parametrize("x,out", [("f16", "e4m3"), ("f32", "f32"), ("bf16", "f16")])
def test_gate_of_many_rows(x, out):
    """2^20 octs and more, two a thread: 517 x 2176 is 128 more than whole
    workgroups take, so the last ones have threads with one oct and with none."""
    rng = np.random.default_rng([len(x), len(out), 1])
    rows, dim = 517, 17408
    both = torch.from_numpy(3 * rng.standard_normal((rows, 2 * dim), np.float32)).to(TORCH[x]).cuda()
    got, scale = room((rows + 1, dim), out)
    q.qtea_silu_mul(both[:, :dim], both[:, dim:], got[:rows], out_scale=None if scale is None else scale[:rows])
    assert (got[rows] == (7 if scale is None else 0x55)).all() and (scale is None or (scale[rows] == 0x55).all())
    some = [0, 1, 120, 240, 241, 482, 515, 516]
    gate, up = both[some, :dim].double().cpu().numpy(), both[some, dim:].double().cpu().numpy()
    want = ol.silu_mul(gate, up)
    check(got[some], None if scale is None else scale[some], want, out, _gate_error(gate, want, out))
    # every row by one that was computed alone
    alone, alone_scale = room((1, dim), out)
    for r in range(0, rows, 37):
        q.qtea_silu_mul(both[r:r + 1, :dim], both[r:r + 1, dim:], alone, out_scale=alone_scale)
        assert torch.equal(alone[0], got[r]) and (scale is None or torch.equal(alone_scale[0], scale[r]))


@pytest.mark.parametrize("rows,dim", [(1, 32), (3, 96), (70, 992)])
def test_gate_of_unaligned_rows_into_8_bits(rows, dim):
    rng = np.random.default_rng([rows, dim])
    both = rounded(2 * rng.standard_normal((rows, 2 * dim + 1)), "f16")
    d = torch.from_numpy(both).half().cuda()
    got, scale = room((rows, dim), "e4m3")
    q.qtea_silu_mul(d[:, 1:1 + dim], d[:, 1 + dim:], got, out_scale=scale)
    gate, up = both[:, 1:1 + dim], both[:, 1 + dim:]
    want = ol.silu_mul(gate, up)
    check(got, scale, want, "e4m3", _gate_error(gate, want, "e4m3"))


# -- the norm --------------------------------------------------------------------------
def _norm_error(t, w, eps):
    """As in tests/test_gpu_layer_rows.py: the addition, sums of up to 64 in a row, a
    wave's 6 steps and its workgroup's 16 (half of them in the root), the factor's four
    roundings and two products."""
    return np.abs(ol.rms_norm(t, w, eps)[0]) * U * (1 + (64 + 6 + 16 + 2) / 2 + 4 + 2)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("residual", [None, "f32", "bf16"])
@pytest.mark.parametrize("out", ["e4m3", "f16"])
@pytest.mark.parametrize("heads,dim", [(7, 96), (3, 128), (5, 512), (2, 1024), (2, 16416)])
def test_norm_of_heads(heads, dim, out, residual, shift):
    """Heads into 8 bits and with a residual, aligned and not: codes, scales and the
    residual of each head at its own place, what lies between tokens as it was."""
    rng = np.random.default_rng([heads, dim, len(out), shift])
    tokens = 5
    X = rounded(rng.standard_normal((tokens, heads, dim)) * 2.0 ** rng.integers(-5, 6, (tokens, heads, 1)), "bf16")
    W = rounded(rng.uniform(0.5, 2, dim), "f32")
    x = torch.zeros((tokens, heads * dim + 8 + shift), dtype=torch.bfloat16, device="cuda")
    x[:, shift:shift + heads * dim] = torch.from_numpy(X).flatten(1).bfloat16()
    R = r = wide_r = None
    if residual:
        R = rounded(rng.standard_normal(X.shape), residual)
        wide_r = torch.full((tokens, (heads + 1) * dim), 7.0, dtype=TORCH[residual], device="cuda")
        r = wide_r[:, :heads * dim].unflatten(1, (heads, dim))
        r.copy_(torch.from_numpy(R))
    got, scale = room((tokens, heads + 1, dim), out)
    q.qtea_rms_norm(x[:, shift:shift + heads * dim].unflatten(1, (heads, dim)), torch.from_numpy(W).float().cuda(), got[:, :heads], residual=r, eps=1e-5,
                    out_scale=None if scale is None else scale[:, :heads])
    want, t = ol.rms_norm(X, W, 1e-5, R)
    check(got[:, :heads], None if scale is None else scale[:, :heads], want, out, _norm_error(t, W, 1e-5))
    assert (got[:, heads] == (7 if scale is None else 0x55)).all() and (scale is None or (scale[:, heads] == 0x55).all())
    if residual:
        assert torch.equal(r.cpu(), (torch.from_numpy(X).float() + torch.from_numpy(R).float()).to(TORCH[residual]))
        assert (wide_r[:, heads * dim:] == 7).all()


@pytest.mark.parametrize("dim", [96, 512, 8192, 16384, 65536])
def test_norm_of_the_largest_and_smallest_values(dim):
    """|t| up to 2^55, and rows whose squares are nothing beside eps."""
    rng = np.random.default_rng(dim)
    X = rounded(rng.choice([-1, 1], (4, dim)) * rng.uniform(0.5, 1, (4, dim)), "f32")
    X *= 2.0 ** np.array([55, 40, -70, -100])[:, None]
    x, out = torch.from_numpy(X).float().cuda(), torch.empty((4, dim), device="cuda")
    q.qtea_rms_norm(x, None, out, eps=1e-30)
    want, t = ol.rms_norm(X, None, float(np.float32(1e-30)))
    check(out, None, want, "f32", _norm_error(t, None, 1e-30))


@pytest.mark.parametrize("shift,pad", [(1, 0), (0, 3)])
@pytest.mark.parametrize("heads,dim", [(1, 96), (5, 128), (3, 256), (1, 4096), (2, 5120), (1, 16384)])
def test_norm_has_the_same_bits_at_any_alignment(heads, dim, shift, pad):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(dim)
    X = torch.randn((9, heads * dim), generator=gen, device="cuda").half()
    wide = torch.zeros((9, heads * dim + shift + pad), dtype=torch.float16, device="cuda")
    wide[:, shift:shift + heads * dim] = X
    a, b = torch.empty((9, heads, dim), device="cuda"), torch.empty((9, heads, dim), device="cuda")
    q.qtea_rms_norm(X.unflatten(1, (heads, dim)), None, a, eps=1e-5)
    q.qtea_rms_norm(wide[:, shift:shift + heads * dim].unflatten(1, (heads, dim)), None, b, eps=1e-5)
    assert torch.equal(a, b)


@pytest.mark.parametrize("rows,dim,x,out", [(8192, 5120, "bf16", "e4m3"), (16, 4096, "f32", "f16"), (3, 1001, "f16", "f32")])
def test_norm_is_the_same_every_time(rows, dim, x, out):
    """The same inputs give the same bits, alone or among other rows."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows)
    X = torch.randn((rows, dim), generator=gen, device="cuda").to(TORCH[x])
    R = torch.randn((rows, dim), generator=gen, device="cuda").to(TORCH[x])
    results = []
    for _ in range(3):
        r, (got, scale) = R.clone(), room((rows, dim), out)
        q.qtea_rms_norm(X, None, got, residual=r, eps=1e-5, out_scale=scale)
        results.append((got, r, scale))
    one, (got, scale) = R[-1:].clone(), room((1, dim), out)
    q.qtea_rms_norm(X[-1:], None, got, residual=one, eps=1e-5, out_scale=scale)
    for other in (*results[1:], None):
        for a, b in zip(results[0], other or (got, one, scale)):
            assert a is None and b is None or torch.equal(a if other else a[-1:], b)


# -- sizes past 2^29 ---------------------------------------------------------------------
def test_gate_of_a_row_past_2_to_the_29():
    dim = 2 ** 29 + 40
    both = torch.empty((1, 2 * dim), dtype=torch.float16, device="cuda")
    both[:, :dim], both[:, dim:] = 1.0, 2.0
    both[0, dim - 1], both[0, -1], both[0, 5] = -2.0, 3.0, 0.0
    out = torch.empty((1, dim), dtype=torch.float16, device="cuda")
    q.qtea_silu_mul(both[:, :dim], both[:, dim:], out)
    one = torch.tensor(2 / (1 + np.exp(-1.0))).half().item()
    assert out[0, 5] == 0 and (out[0, 6:-1] == one).all() and abs(out[0, -1].item() + 6 / (1 + np.exp(2.0))) < 1e-3


def test_norm_of_a_token_past_2_to_the_29():
    heads, dim = 65535, 8224
    assert heads * dim > 2 ** 29
    x = torch.ones((2, heads, dim), dtype=torch.float16, device="cuda")
    x[1, -1] = 4.0
    x[1, -1, ::2] = -2.0
    q.qtea_rms_norm(x, None, x, eps=1e-6)
    want = torch.tensor([-2.0, 4.0]).div(10 ** 0.5).half().cuda()
    assert (x[0] == 1).all() and (x[1, :-1] == 1).all() and torch.equal(x[1, -1, :2], want) and torch.equal(x[1, -1, -2:], want)


@pytest.mark.parametrize("batch,offset", [(1, 0), (3, 0), (2, 1)])
def test_product_of_more_than_2_to_the_29_rows(batch, offset):
    """The packed matrix of up to 128 columns has one tile a strip, strip after strip, then
    their scales: zeros, with the first and the last strips' from a small one."""
    N, K = 2 ** 29 + 19, 40
    strips = -(-N // 16)
    m = q.W4Matrix(N, K, torch.zeros(q.qtea_w4_packed_bytes(N, K), dtype=torch.uint8, device="cuda"))
    assert m.packed.numel() == strips * 1280
    small = torch.zeros((32, K), device="cuda")
    small[0, 3], small[16 + (N - 1) % 16, K - 1], small[16, 0] = 3.0, 1.5, -2.0
    packed = q.pack_matrix_w4(small).packed
    m.packed[strips * 1024:] = packed[2048 + 8]  # (a scale byte of zeros)
    for at, strip in ((0, 0), (1, strips - 1)):
        m.packed[strip * 1024:(strip + 1) * 1024] = packed[at * 1024:(at + 1) * 1024]
        m.packed[strips * 1024 + strip * 256:strips * 1024 + (strip + 1) * 256] = packed[2048 + at * 256:2048 + (at + 1) * 256]
    X = torch.zeros((batch, K + 2 * offset), dtype=torch.float16, device="cuda")[:, offset:offset + K]
    X[:] = torch.arange(1, batch + 1, device="cuda")[:, None].half()
    Y = torch.full((batch, N), 7.0, dtype=torch.float16, device="cuda")
    q.qtea_w4_gemm_lowbatch(m, X, Y)
    for b in range(batch):
        y = Y[b]
        assert y[0] == 3 * (b + 1) and y[-1] == 1.5 * (b + 1) and y[(strips - 1) * 16] == -2 * (b + 1)
        assert int((y != 0).sum()) == 3


# -- the rotation ------------------------------------------------------------------------
def _turn_error(x, pos, freq, interleaved):
    """Sine and cosine are found in 64 bits, to a tenth of half an ulp of fp32 at any angle
    (and 2^-50 next to their zeros), and rounded once; the two products are rounded
    once each.  So |a cos| and |b sin| are off by 2.1 U of themselves; their sum's
    rounding is the result's."""
    half = len(freq)
    angle = np.asarray(pos, np.longdouble)[:, None] * np.asarray(freq, np.longdouble)
    cos, sin = np.abs(np.cos(angle)).astype(np.float64)[:, None], np.abs(np.sin(angle)).astype(np.float64)[:, None]
    a, b = (np.arange(half) * 2, np.arange(half) * 2 + 1) if interleaved else (np.arange(half), np.arange(half) + half)
    x, err = np.abs(x), np.zeros_like(x)
    err[..., a], err[..., b] = x[..., a] * cos + x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    return 2.2 * U * err + 2.0 ** -48 * x.max(-1, keepdims=True)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("context,base", [(40, 1.0), (5000, 1e4), (1 << 24, 5e5), (524285 * 4096, 1e6)])
def test_rotated_to_the_last_bits(context, base, interleaved):
    """Angles up to 2^51 (frequencies up to 2^20), each pair to three half ulps of its parts."""
    rng = np.random.default_rng([context % 1000, interleaved])
    n, heads, dim, page = 24, 3, 128, 4096
    max_pages = -(-context // page)
    table = torch.full((1, max_pages), -1, dtype=torch.int32, device="cuda")
    first = (context - n) // page
    table[0, first:] = torch.arange(max_pages - first, device="cuda")
    cache = q.new_kv_cache("f16", max_pages - first, page, 1, dim)
    Q = rounded(rng.standard_normal((n, heads, dim)) * 2.0 ** rng.integers(-20, 20, (n, heads, 1)), "f32")
    freq = (base ** (-2.0 * np.arange(dim // 2) / dim)).astype(np.float32)
    freq[1::7] = rng.uniform(0.3, 7, freq[1::7].shape)
    freq[2::7] = -rng.uniform(0.5, 1, freq[2::7].shape) * 2.0 ** rng.integers(0, 21, freq[2::7].shape)
    freq[3::28] = 0
    x = torch.from_numpy(Q).float().cuda()
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    out = torch.empty_like(x)
    q.qtea_kv_append_rotated(cache, x, x[:, :1], x[:, 1:2], i32(0, n), i32(context), table, torch.from_numpy(freq).cuda(), out, interleaved=interleaved)
    pos = np.arange(context - n, context)
    check(out, None, ol.rotate(Q, pos, freq, interleaved), "f32", _turn_error(Q, pos, freq, interleaved))
