"""Matrices of 4-bit codes: packing bit for bit, products against 64 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.layer as ol
import oracle.serving as sv
import paper_2609_00224_amd as q
from tests.layer_cases import HALF, TINY, TORCH, rounded

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (16, 128), (17, 129), (33, 1000), (1000, 256), (130, 4128), (48, 14336), (5, 40000), (700, 511), (2049, 640)]


def _dev(x, kind):
    return torch.from_numpy(np.ascontiguousarray(x)).to(TORCH[kind]).cuda()


@pytest.mark.parametrize("kind", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (17, 129), (33, 1000), (50, 513), (3, 31)])
def test_pack_is_the_oracles_and_packing_again_changes_nothing(N, K, kind):
    rng = np.random.default_rng([N, K])
    mag = np.repeat(2.0 ** rng.integers(-14, 12, (N, -(-K // 32))), 32, 1)[:, :K]
    W = rng.standard_normal((N, K)) * mag
    W[rng.random((N, K)) < 0.1] = 0
    tie = rng.random((N, K)) < 0.2
    W = rounded(np.where(tie, np.round(rng.uniform(-24, 24, (N, K))) * 0.25 * mag, W), kind)
    # rows of a wider tensor
    wide = torch.zeros((N, K + 3), dtype=TORCH[kind], device="cuda")
    wide[:, 1:1 + K] = _dev(W, kind)
    m = q.pack_matrix_w4(wide[:, 1:1 + K])
    want = ol.w4_values(W)
    for to in ("f16", "bf16", "f32"):
        room = torch.full((N, K + 5), 7.0, dtype=TORCH[to], device="cuda")
        q.qtea_w4_unpack(m, room[:, 2:2 + K])
        assert np.array_equal(room[:, 2:2 + K].double().cpu().numpy(), want)
        assert (room[:, :2] == 7).all() and (room[:, 2 + K:] == 7).all()
    again = q.pack_matrix_w4(_dev(want, "f16"))
    out = torch.empty((N, K), device="cuda")
    q.qtea_w4_unpack(again, out)
    assert np.array_equal(out.double().cpu().numpy(), want)


def _acts(rng, batch, K, x):
    """Activations: (values, X, x_scale)."""
    v = rng.standard_normal((batch, K)) * 2.0 ** rng.integers(-3, 4, (batch, 1))
    if x != "e4m3":
        v = rounded(v, x)
        return v, _dev(v, x), None
    code, scale = sv.encode(v, "e4m3")
    return sv.decode(code, scale, "e4m3"), torch.from_numpy(code).cuda(), torch.from_numpy(scale).cuda()


@pytest.mark.parametrize("x,y", [("f16", "f32"), ("bf16", "f32"), ("e4m3", "f32"), ("f16", "f16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("batch", [1, 3, 16, 17, 40, 64])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_product(case, batch, x, y):
    N, K = SHAPES[case]
    if x == "e4m3":
        K = -(-K // 32) * 32
    rng = np.random.default_rng([case, batch, len(x)])
    W = ol.w4_values(rng.standard_normal((N, K)) * K ** -0.5)
    v, X, xs = _acts(rng, batch, K, x)
    room = torch.full((batch + 1, N + 3), 7.0, dtype=TORCH[y], device="cuda")
    q.qtea_w4_gemm_lowbatch(q.pack_matrix_w4(_dev(W, "f16")), X, room[:batch, :N], x_scale=xs)
    got, want = room[:batch, :N].double().cpu().numpy(), v @ W.T
    assert (room[batch:] == 7).all() and (room[:, N:] == 7).all()
    # exact products; K additions, each off by at most 2^-23 (a truncation) of
    # the largest partial sum; one rounding
    bound = K * 2.0 ** -23 * (np.abs(v) @ np.abs(W).T)
    bound = bound + HALF[y] * (np.abs(want) + bound) + TINY[y]
    assert (np.abs(got - want) <= bound).all()
    # errors of either sign: the root of their number, in the mean
    if N * batch >= 100:
        assert np.linalg.norm(got - want) <= np.linalg.norm(want) * (2.0 ** -23 * K ** 0.5 + HALF[y])


@pytest.mark.parametrize("x", ["f16", "bf16", "e4m3"])
@pytest.mark.parametrize("batch", [1, 2, 5, 16, 33, 64])
@pytest.mark.parametrize("N,K", [(16, 32), (77, 1024), (100, 2208), (1030, 96), (19, 8224)])
def test_whole_numbers_are_exact(N, K, batch, x):
    """Halves and whole numbers whose sums stay below 2^23 halves: every column
    meets its own weight."""
    rng = np.random.default_rng([N, K, batch])
    W = rng.choice([0, 0.5, 1, 1.5, 2, 3, 4, 6], (N, K)) * rng.choice([-1, 1], (N, K)) * 2.0 ** np.repeat(rng.integers(0, 3, (N, K // 32)), 32, 1)
    v = rng.integers(-8, 9, (batch, K)).astype(np.float64)
    if x == "e4m3":
        code, scale = sv.encode(v, "e4m3")
        assert np.array_equal(sv.decode(code, scale, "e4m3"), v)
        X, xs = torch.from_numpy(code).cuda(), torch.from_numpy(scale).cuda()
    else:
        X, xs = _dev(v, x), None
    Y = torch.empty((batch, N), device="cuda")
    q.qtea_w4_gemm_lowbatch(q.pack_matrix_w4(_dev(W, "f32")), X, Y, x_scale=xs)
    assert np.array_equal(Y.double().cpu().numpy(), v @ W.T)


@pytest.mark.parametrize("x", ["f16", "bf16", "e4m3"])
@pytest.mark.parametrize("batch", [1, 8, 16, 17, 32, 33, 48, 64])
@pytest.mark.parametrize("N,K", [(12290, 96), (20481, 32), (20500, 544), (32000, 160), (61440, 1056), (131073, 64)])
def test_many_rows_of_weights(N, K, batch, x):
    """Five and more strips of 16 rows a CU (three past 16 rows of X): every
    count of strips a wave takes, a unit of columns and more; exact sums."""
    rng = np.random.default_rng([N, K, batch])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N + batch)
    steps = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    W = steps[torch.randint(0, 15, (N, K), generator=gen, device="cuda")]
    v = rng.integers(-8, 9, (batch, K)).astype(np.float64)
    X, xs = _dev(v, "f16" if x == "e4m3" else x), None
    if x == "e4m3":
        code, scale = sv.encode(v, "e4m3")
        X, xs = torch.from_numpy(code).cuda(), torch.from_numpy(scale).cuda()
    room = torch.full((batch + 1, N + 3), 7.0, device="cuda")
    q.qtea_w4_gemm_lowbatch(q.pack_matrix_w4(W), X, room[:batch, :N], x_scale=xs)
    want = torch.from_numpy(v).float().cuda() @ W.T  # whole halves below 2^24: exact in any order
    assert torch.equal(room[:batch, :N], want)
    assert (room[batch:] == 7).all() and (room[:, N:] == 7).all()


@pytest.mark.parametrize("x", ["f16", "bf16", "e4m3"])
@pytest.mark.parametrize("batch", [1, 17, 33, 64])
@pytest.mark.parametrize("N,K", [(57330, 4896), (65540, 4224), (128257, 2112)])
def test_matrices_that_no_cache_keeps(N, K, batch, x):
    """More than 128 MB of codes, 16, 8 and 32 strips a workgroup; exact sums."""
    assert q.qtea_w4_packed_bytes(N, K) * 16 // 17 > 128 << 20
    test_many_rows_of_weights(N, K, batch, x)


@pytest.mark.parametrize("N", [90, 24000])
@pytest.mark.parametrize("K,shift,pad", [(1000, 0, 8), (1000, 1, 0), (999, 0, 0), (1024, 3, 2), (4096, 0, 1), (130, 5, 6)])
def test_rows_of_any_stride(K, shift, pad, N):
    rng = np.random.default_rng([K, shift])
    W = rng.choice([0, 0.5, 1, 3], (N, K))
    v = rng.integers(-4, 5, (7, K)).astype(np.float64)
    wide = torch.full((7, shift + K + pad), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, shift:shift + K] = _dev(v, "f16")
    Y = torch.empty((7, N), device="cuda")
    q.qtea_w4_gemm_lowbatch(q.pack_matrix_w4(_dev(W, "f16")), wide[:, shift:shift + K], Y)
    assert np.array_equal(Y.double().cpu().numpy(), v @ W.T)


def test_strided_codes():
    rng = np.random.default_rng(8)
    W, v = rng.choice([0, 0.5, 1, 3], (40, 96)), rng.integers(-4, 5, (5, 96)).astype(np.float64)
    code, scale = sv.encode(v, "e4m3")
    X = torch.full((5, 160), 0x7f, dtype=torch.uint8, device="cuda")
    xs = torch.full((5, 7), 255, dtype=torch.uint8, device="cuda")
    X[:, 32:128], xs[:, 2:5] = torch.from_numpy(code).cuda(), torch.from_numpy(scale).cuda()
    Y = torch.empty((5, 40), device="cuda")
    q.qtea_w4_gemm_lowbatch(q.pack_matrix_w4(_dev(W, "f16")), X[:, 32:128], Y, x_scale=xs[:, 2:5])
    assert np.array_equal(Y.double().cpu().numpy(), v @ W.T)


def test_the_formats_range():
    """The smallest and largest exponents of a block, in every type of activation."""
    W = np.zeros((3, 96))
    W[0, 0], W[0, 40], W[1, 5], W[2, 70] = 2.0 ** -24, 6 * 2.0 ** 13, 1.5 * 2.0 ** -23, -(2.0 ** 15)
    m = q.pack_matrix_w4(_dev(W, "f32"))
    for x in ("f16", "bf16", "e4m3"):
        v = np.zeros((3, 96))
        v[0, 0], v[1, 40], v[2, 5], v[0, 70] = 2, 1, 1, 0.5
        X, xs = _dev(v, x if x != "e4m3" else "f32"), None
        if x == "e4m3":
            code, scale = sv.encode(v, "e4m3")
            X, xs = torch.from_numpy(code).cuda(), torch.from_numpy(scale).cuda()
        Y = torch.empty((3, 3), device="cuda")
        q.qtea_w4_gemm_lowbatch(m, X, Y, x_scale=xs)
        assert np.array_equal(Y.double().cpu().numpy(), v @ W.T), x


@pytest.mark.parametrize("byte", [10, 60, 127, 200, 246])
def test_scales_of_the_activations(byte):
    """The smallest and largest codes times the smallest and largest scales that are exact."""
    W = np.zeros((2, 64))
    W[0, 3], W[1, 33], W[1, 34] = 0.5, 1, -0.5
    X = torch.zeros((3, 64), dtype=torch.uint8, device="cuda")
    X[0, 3], X[1, 33], X[2, 33], X[2, 34] = 0x01, 0x7e, 0x81, 0xfe
    xs = torch.full((3, 2), byte, dtype=torch.uint8, device="cuda")
    Y = torch.empty((3, 2), device="cuda")
    q.qtea_w4_gemm_lowbatch(q.pack_matrix_w4(_dev(W, "f32")), X, Y, x_scale=xs)
    v = sv.decode(X.cpu().numpy(), xs.cpu().numpy(), "e4m3")
    assert np.array_equal(Y.double().cpu().numpy(), (v @ W.T).astype(np.float32).astype(np.float64))


@pytest.mark.parametrize("x", ["f16", "bf16", "e4m3"])
def test_what_is_not_finite_stays_in_its_row(x):
    rng = np.random.default_rng(9)
    W = rng.choice([0.5, 1, 3], (40, 256))
    W[7, 100] = np.nan  # a block of row 7
    v = rng.integers(1, 5, (18, 256)).astype(np.float64)
    v[3, 200], v[17, 9] = np.nan, np.inf
    if x == "e4m3":
        code, scale = sv.encode(v, "e4m3")
        X, xs = torch.from_numpy(code).cuda(), torch.from_numpy(scale).cuda()
    else:
        X, xs = _dev(v, x), None
    Y = torch.empty((18, 40), device="cuda")
    q.qtea_w4_gemm_lowbatch(q.pack_matrix_w4(_dev(W, "f32")), X, Y, x_scale=xs)
    Y = Y.double().cpu().numpy()
    assert np.isnan(Y[:, 7]).all() and np.isnan(Y[3]).all()
    rest = np.delete(np.delete(Y, 7, 1), [3, 17], 0)
    assert np.array_equal(rest, np.delete(np.delete(v, [3, 17], 0) @ W.T, 7, 1))
    assert (np.isnan(np.delete(Y[17], 7)) if x == "e4m3" else np.delete(Y[17], 7) == np.inf).all()


def test_on_a_stream_of_its_own_in_a_graph_and_twice_the_same():
    rng = np.random.default_rng(10)
    W = ol.w4_values(rng.standard_normal((500, 1500)))
    m = q.pack_matrix_w4(_dev(W, "f16"))
    X = torch.randn((9, 1500), device="cuda").half()
    Y, Z = torch.empty((9, 500), device="cuda"), torch.empty((9, 500), device="cuda")
    q.qtea_w4_gemm_lowbatch(m, X, Y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q.qtea_w4_gemm_lowbatch(m, X, Z, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(Y, Z)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        q.qtea_w4_gemm_lowbatch(m, X, Z)
    for i in range(4):
        X.copy_(torch.randn(X.shape, device="cuda"))
        g.replay()
        q.qtea_w4_gemm_lowbatch(m, X, Y)
        torch.cuda.synchronize()
        assert torch.equal(Y, Z)


def test_no_rows():
    m = q.pack_matrix_w4(torch.ones((5, 40), device="cuda"))
    q.qtea_w4_gemm_lowbatch(m, torch.empty((0, 40), dtype=torch.float16, device="cuda"), torch.empty((0, 5), device="cuda"))


def test_codes_past_32_bits():
    """A packed matrix of more than 2^32 bytes: its last rows."""
    N, K = 300003, 28704
    m = q.W4Matrix(N, K, torch.zeros(q.qtea_w4_packed_bytes(N, K), dtype=torch.uint8, device="cuda"))
    assert m.packed.numel() > 1 << 32
    W = torch.zeros((N, K), dtype=torch.float16, device="cuda")
    W[-1, -1], W[-2, 3], W[0, 5] = 3, 0.5, 6
    q.qtea_w4_pack(W, m.packed)
    del W
    X = torch.ones((2, K), dtype=torch.float16, device="cuda")
    X[1] = 2
    Y = torch.empty((2, N), device="cuda")
    q.qtea_w4_gemm_lowbatch(m, X, Y)
    want = torch.zeros((2, N), device="cuda")
    want[:, -1], want[:, -2], want[:, 0] = 3, 0.5, 6
    want[1] *= 2
    assert torch.equal(Y, want)
