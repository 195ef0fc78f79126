"""qtea_rms_norm and qtea_silu_mul against their definitions in 64 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.layer as ol
import paper_2609_00224_amd as q
from tests.layer_cases import TORCH, U, check, room, rounded

pytestmark = pytest.mark.gpu

# rows, dim: every count of threads a row can have, rows that fill no workgroup, odd lengths
SHAPES = [(1, 1), (3, 7), (5, 32), (9, 64), (70, 96), (33, 128), (2, 200), (17, 512), (3, 1001), (6, 1024), (2, 2048), (1, 4096), (5, 4095),
          (4, 5120), (3, 8192), (2, 14336), (1, 16384), (2, 20001), (1, 40000), (1, 65536)]


def _norm_error(t, w, dim, eps):
    """What fp32 may be off in t / sqrt(mean + eps) * w: the addition (1/2 ulp
    of t), a sum of squares of at most 64 values in a row, 6 steps over a
    wave and 16 over its workgroup's waves (half of that in the root), four more
    roundings to the factor and two products."""
    y = np.abs(ol.rms_norm(t, w, eps)[0])
    return y * U * (1 + (64 + 6 + 16 + 2) / 2 + 4 + 2)


def _put(x, kind, pad=0, shift=0):
    """x [rows][...] on the device: rows `pad` elements further apart, `shift` from an aligned start."""
    flat = torch.from_numpy(np.ascontiguousarray(x)).reshape(x.shape[0], -1).to(TORCH[kind])
    wide = torch.zeros((x.shape[0], flat.shape[1] + pad + shift), dtype=TORCH[kind], device="cuda")
    view = wide[:, shift:shift + flat.shape[1]]
    view.copy_(flat)
    return view if x.ndim == 2 else view.unflatten(1, x.shape[1:])


@pytest.mark.parametrize("x,res,w,out", [("f32", "f32", "f32", "f16"), ("f16", "bf16", "f16", "bf16"), ("bf16", "f16", "bf16", "f32"), ("f16", None, None, "f16"),
                                         ("bf16", "bf16", "bf16", "e4m3"), ("f32", None, "f32", "e4m3"), ("f32", "f16", None, "bf16")])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_norm(case, x, res, w, out):
    rows, dim = SHAPES[case]
    if out == "e4m3":
        dim = -(-dim // 32) * 32
    rng = np.random.default_rng([case, len(x), len(out)])
    X = rounded(rng.standard_normal((rows, dim)) * 2.0 ** rng.integers(-6, 7, (rows, 1)), x)
    R = None if res is None else rounded(rng.standard_normal((rows, dim)), res)
    W = None if w is None else rounded(rng.uniform(0.2, 3, dim), w)
    got, scale = room((rows, dim), out)
    rd = None if R is None else _put(R, res)
    q.qtea_rms_norm(_put(X, x), None if W is None else torch.from_numpy(W).to(TORCH[w]).cuda(), got, residual=rd, eps=1e-5, out_scale=scale)
    want, t = ol.rms_norm(X, W, 1e-5, R)
    check(got, scale, want, out, _norm_error(t, W, dim, 1e-5))
    if R is not None:  # the fp32 sum, rounded
        assert torch.equal(rd.cpu(), (torch.from_numpy(X).float() + torch.from_numpy(R).float()).to(TORCH[res]))


@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (3, 1), (0, 4)])
@pytest.mark.parametrize("dim", [40, 96, 1000, 4096])
def test_norm_of_strided_and_unaligned_rows(dim, pad, shift):
    rng = np.random.default_rng([dim, pad, shift])
    X, R = (rounded(rng.standard_normal((5, dim)), "f16") for _ in range(2))
    x, r = _put(X, "f16", pad, shift), _put(R, "f16", shift, pad)
    wide = torch.full((5, dim + pad + 9), 7.0, dtype=torch.float16, device="cuda")
    out = wide[:, 1:1 + dim]
    q.qtea_rms_norm(x, None, out, residual=r, eps=1e-6)
    want, t = ol.rms_norm(X, None, 1e-6, R)
    check(out, None, want, "f16", _norm_error(t, None, dim, 1e-6))
    assert (wide[:, 0] == 7).all() and (wide[:, 1 + dim:] == 7).all()
    assert torch.equal(r.cpu(), torch.from_numpy(t).half())


@pytest.mark.parametrize("heads,dim", [(1, 64), (5, 64), (7, 96), (40, 128), (3, 256), (2, 1000)])
def test_norm_of_heads_where_they_are(heads, dim):
    """The query heads of a fused projection's output, in place; its other columns stay."""
    rng = np.random.default_rng([heads, dim])
    X = rounded(rng.standard_normal((11, heads + 2, dim)), "bf16")
    W = rounded(rng.uniform(0.5, 2, dim), "bf16")
    x = _put(X, "bf16")
    view = x[:, 1:1 + heads]
    q.qtea_rms_norm(view, torch.from_numpy(W).bfloat16().cuda(), view, eps=1e-6)
    want, t = ol.rms_norm(X[:, 1:1 + heads], W, 1e-6)
    check(view, None, want, "bf16", _norm_error(t, W, dim, 1e-6))
    assert torch.equal(x[:, 0].cpu().double(), torch.from_numpy(X[:, 0])) and torch.equal(x[:, -1].cpu().double(), torch.from_numpy(X[:, -1]))


def test_norm_of_zeros_infinities_and_nan():
    x = torch.ones((5, 256), device="cuda")
    x[0] = 0
    x[1, 3], x[2, 40], x[3, 255] = float("inf"), float("nan"), float("-inf")
    out, scale = room((5, 256), "e4m3")
    dense = torch.empty_like(x)
    q.qtea_rms_norm(x, None, dense, eps=1e-6)
    q.qtea_rms_norm(x, None, out, eps=1e-6, out_scale=scale)
    assert (dense[0] == 0).all() and (out[0] == 0).all()
    # an infinity takes the others to 0 and itself to NaN, a NaN the whole row
    assert dense[1].isnan().sum() == 1 and dense[1, 3].isnan() and dense[3].isnan().sum() == 1 and dense[2].isnan().all()
    nan = (scale == 255).cpu()
    assert nan[1].tolist() == [True] + [False] * 7 and nan[3].tolist() == [False] * 7 + [True] and nan[2].all() and not nan[0].any() and not nan[4].any()
    assert torch.allclose(dense[4], torch.ones(256, device="cuda"), atol=1e-5)


@pytest.mark.parametrize("x,out", [("f32", "f16"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("f32", "e4m3")])
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 7), (1, 32), (130, 96), (16, 14336), (3, 4099), (2, 28672)])
def test_gate(rows, dim, x, out):
    if out == "e4m3":
        dim = -(-dim // 32) * 32
    rng = np.random.default_rng([rows, dim, len(x)])
    both = rounded(rng.standard_normal((rows, 2 * dim)) * rng.choice([0.1, 1, 30], (rows, 2 * dim)), x)
    d = torch.from_numpy(both).to(TORCH[x]).cuda()
    got, scale = room((rows, dim), out)
    q.qtea_silu_mul(d[:, :dim], d[:, dim:], got, out_scale=scale)
    want = ol.silu_mul(both[:, :dim], both[:, dim:])
    # exp: 2 ulp, the sum, the quotient and the product half an ulp each; a
    # gate below -88 gives 0 for less than 88 exp(-88)
    check(got, scale, want, out, 8 * U * np.abs(want) + 2.0 ** -118 * np.abs(both[:, dim:]))


def test_gate_in_place_and_strided():
    rng = np.random.default_rng(4)
    both = rounded(rng.standard_normal((9, 301)), "f16")
    for shift in (0, 1):
        d = torch.from_numpy(both).half().cuda()
        gate, up = d[:, shift:shift + 120], d[:, 150 + shift:270 + shift]
        q.qtea_silu_mul(gate, up, gate if shift else up)
        want = ol.silu_mul(both[:, shift:shift + 120], both[:, 150 + shift:270 + shift])
        check(gate if shift else up, None, want, "f16", 8 * U * np.abs(want))
        kept = torch.from_numpy(both).half().cuda()
        kept[:, shift:shift + 120] = gate
        kept[:, 150 + shift:270 + shift] = up
        assert torch.equal(d, kept)


def test_gate_of_infinities_and_nan():
    g = torch.tensor([[0.0, float("inf"), float("-inf"), float("nan"), 1.0, -200.0, 200.0, 3.0]], device="cuda")
    u = torch.tensor([[float("inf"), 2.0, 2.0, 2.0, float("nan"), 5.0, 5.0, float("-inf")]], device="cuda")
    out = torch.empty_like(g)
    q.qtea_silu_mul(g, u, out)
    assert torch.equal(out.isnan().cpu()[0], torch.tensor([1, 0, 1, 1, 1, 0, 0, 0]).bool())
    assert out[0, 1] == float("inf") and out[0, 5] == 0 and out[0, 6] == 1000 and out[0, 7] == float("-inf")


def test_rows_on_a_stream_of_their_own_and_in_a_graph():
    x, r, out = torch.zeros((6, 4096), device="cuda"), torch.zeros((6, 4096), device="cuda"), torch.empty((6, 4096), dtype=torch.float16, device="cuda")
    codes, scale = room((6, 2048), "e4m3")

    def step(stream=None):
        q.qtea_rms_norm(x, None, out, residual=r, eps=1e-6, stream=stream)
        q.qtea_silu_mul(out[:, :2048], out[:, 2048:], codes, out_scale=scale, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert (out == 0).all() and (codes == 0).all()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        x.copy_(torch.randn(x.shape, device="cuda"))
        before = r.clone()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, r, codes, scale)]
        r.copy_(before)
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, r, codes, scale)))


def test_no_rows():
    z = torch.empty((0, 64), device="cuda")
    q.qtea_rms_norm(z, None, z.half())
    q.qtea_silu_mul(z, z, z.half())


def test_rows_past_32_bits():
    """More than 2^32 elements: the last rows."""
    rows, dim = 65540, 65536
    x = torch.ones((rows, dim), dtype=torch.bfloat16, device="cuda")
    x[-1] = 2
    x[-1, ::2] = -4
    q.qtea_rms_norm(x, None, x, eps=1e-6)
    assert (x[0] == 1).all() and (x[65536] == 1).all()
    want = torch.tensor([-4, 2]).div(10 ** 0.5).bfloat16().cuda()
    assert torch.equal(x[-1, :2], want) and torch.equal(x[-1, -2:], want)
    del x
    both = torch.ones((rows, 65536), dtype=torch.bfloat16, device="cuda")
    both[-1] = 2
    q.qtea_silu_mul(both[:, :32768], both[:, 32768:], both[:, 32768:])
    assert torch.allclose(both[-1, 32768:].float(), torch.tensor(4 / (1 + np.exp(-2.0)), device="cuda").float(), rtol=2 ** -8)
    assert (both[-1, :32768] == 2).all()
