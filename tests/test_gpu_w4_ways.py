"""Products with 4-bit weights along each way that sizes lead to on 256 CUs:
exact sums, so that every code, scale and activation has to meet its own."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.serving as sv
import paper_2609_00224_amd as q
from tests.layer_cases import TORCH

pytestmark = pytest.mark.gpu

STEPS = (0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.5, -1, -1.5, -2, -3, -4, -6)

# N, K, batches, activations.  A strip is 16 rows of weights, a unit 512 columns.
FEW = [
    # four strips a group, eight waves share a group's columns: units of each 1..2, 0..1, 4..5, 2..3
    (4099, 4128, (40, 64), ("f16", "bf16", "e4m3")),
    (10243, 2600, (1, 3, 8, 16), ("f16", "bf16")),
    (10243, 2592, (1, 3, 8, 16), ("e4m3",)),
    (10260, 17440, (4, 16), ("f16", "e4m3")),
    (5123, 8224, (17, 40), ("f16", "bf16", "e4m3")),
    # two strips a group: 2..3 and 4..5 units
    (5123, 8224, (1, 3, 8, 16), ("f16", "bf16", "e4m3")),
    (5130, 17440, (5, 16), ("bf16", "e4m3")),
    # one strip: 6..7
    (2050, 26656, (2, 16, 31), ("f16", "e4m3")),
    # rows of X that are not 4-byte aligned (odd K): one, two, four and eight waves a
    # group of two strips, each with several units
    (65555, 1301, (1, 7), ("f16",)),
    (32787, 2601, (1, 18), ("bf16",)),
    (16410, 4127, (3, 16), ("f16",)),
    (5123, 8225, (16, 33), ("f16",)),
]
# many strips: 32, 16 and 8 a workgroup with codes that the caches keep, up to six units
MANY = [
    (128257, 1056, (1, 16, 17, 33, 64), ("f16", "bf16", "e4m3")),
    (57330, 2600, (1, 16, 40), ("f16", "bf16")),
    (57330, 2592, (5, 64), ("e4m3",)),
    (28675, 2600, (1, 8, 16, 32, 48, 64), ("f16", "bf16")),
    (28675, 2592, (1, 16, 33), ("e4m3",)),
]


def _flat(cases):
    return [(N, K, b, x) for N, K, batches, types in cases for b in batches for x in types]


def _whole(N, K, batch, x, seed):
    """Weights in halves up to 24 with every block's scale one of three, and
    activations in whole numbers up to 32, a block's scale one of three: W, v (fp32 on
    the device) and X, x_scale."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    blocks = -(-K // 32)
    by = lambda rows: 2.0 ** torch.randint(0, 3, (rows, blocks), generator=gen, device="cuda").float().repeat_interleave(32, 1)[:, :K]  # noqa: E731
    W = torch.tensor(STEPS, device="cuda")[torch.randint(0, len(STEPS), (N, K), generator=gen, device="cuda")] * by(N)
    v = torch.randint(-8, 9, (batch, K), generator=gen, device="cuda").float() * by(batch)
    if x != "e4m3":
        return W, v, v.to(TORCH[x]), None
    code, scale = sv.encode(v.double().cpu().numpy(), "e4m3")
    assert np.array_equal(sv.decode(code, scale, "e4m3"), v.double().cpu().numpy())
    return W, v, torch.from_numpy(code).cuda(), torch.from_numpy(scale).cuda()


@pytest.mark.parametrize("N,K,batch,x", _flat(FEW) + _flat(MANY))
def test_every_way_is_exact(N, K, batch, x):
    W, v, X, xs = _whole(N, K, batch, x, N + K + batch)
    room = torch.full((batch + 1, N + 3), 7.0, device="cuda")
    q.qtea_w4_gemm_lowbatch(q.pack_matrix_w4(W), X, room[:batch, :N], x_scale=xs)
    # in halves, below 2^24 of them wherever the signs are not all one: in 64 bits
    want = torch.empty((batch, N), dtype=torch.float64, device="cuda")
    for at in range(0, N, 8192):
        want[:, at:at + 8192] = v.double() @ W[at:at + 8192].double().T
    assert float((v.abs() @ W.abs()[:4096].T).max()) < 2.0 ** 23
    assert torch.equal(room[:batch, :N].double(), want)
    assert (room[batch:] == 7).all() and (room[:, N:] == 7).all()


@pytest.mark.parametrize("y", ["f16", "bf16"])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("N,K,batch,x", [(28675, 544, 16, "f16"), (20484, 96, 40, "e4m3"), (128257, 96, 3, "bf16"), (5123, 8224, 16, "f16"), (4099, 4128, 40, "bf16")])
def test_results_of_16_bits(N, K, batch, x, pad, y):
    """Exact sums, rounded once: small enough for fp16 by a power of two at the activations."""
    W, v, X, xs = _whole(N, K, batch, x, N + batch)
    if xs is None:
        X = X * 2.0 ** -8
    else:
        xs = xs - 8
    room = torch.full((batch, N + pad), 7.0, dtype=TORCH[y], device="cuda")
    q.qtea_w4_gemm_lowbatch(q.pack_matrix_w4(W), X, room[:, :N], x_scale=xs)
    want = torch.empty((batch, N), dtype=torch.float64, device="cuda")
    for at in range(0, N, 8192):
        want[:, at:at + 8192] = v.double() @ W[at:at + 8192].double().T * 2.0 ** -8
    assert torch.equal(room[:, :N], want.float().to(TORCH[y]))  # (exact in fp32)
    assert (room[:, N:] == 7).all()


@pytest.mark.parametrize("x", ["f16", "bf16", "e4m3"])
@pytest.mark.parametrize("N,K,batch", [(20489, 2592, 18), (57330, 96, 18), (128257, 96, 18), (28675, 1056, 64), (5123, 8224, 18), (10243, 2592, 16)])
def test_what_is_not_finite_stays_in_its_row(N, K, batch, x):
    """NaN blocks of weights in the first and last strips and the last columns, NaN and
    infinities of activations: their own results only."""
    W, v, X, xs = _whole(N, K, batch, x, N + 1)
    rows, cols = [0, 17, N // 2, N - 1], [0, min(511, K - 2), K - 33, K - 1]
    W[rows, cols] = float("nan")
    m = q.pack_matrix_w4(W)
    bad = [3, batch - 1]
    if x == "e4m3":
        xs[3, K // 32 - 1], xs[batch - 1, 0] = 255, 255
    else:
        X[3, K - 1], X[batch - 1, 0] = float("nan"), float("nan")
    Y = torch.empty((batch, N), device="cuda")
    q.qtea_w4_gemm_lowbatch(m, X, Y, x_scale=xs)
    assert Y[:, rows].isnan().all() and Y[bad].isnan().all()
    keep, good = torch.ones(N, dtype=torch.bool, device="cuda"), [b for b in range(batch) if b not in bad]
    keep[rows] = False
    W[rows] = 0
    for at in range(0, N, 8192):
        want = v[good].double() @ W[at:at + 8192].double().T
        assert torch.equal(Y[good, at:at + 8192].double()[:, keep[at:at + 8192]], want[:, keep[at:at + 8192]])


@pytest.mark.parametrize("N,K,batch", [(70, 640, 3), (5123, 8224, 8), (28675, 544, 16), (128257, 544, 33)])
def test_the_formats_range(N, K, batch):
    """The smallest and largest values of blocks and activations (fp16's smallest
    numbers among them), on every way: one product a result."""
    W = torch.zeros((N, K), device="cuda")
    at = {0: (0, 2.0 ** -24), N - 1: (K - 1, 6 * 2.0 ** 13), N // 2: (33, 1.5 * 2.0 ** -23), 9: (K - 70, -(2.0 ** 15))}
    for n, (k, w) in at.items():
        W[n, k] = w
    m = q.pack_matrix_w4(W)
    for x, values in (("f16", (2.0, 1.0, -(2.0 ** -24), 1023 * 2.0 ** -24, 2.0 ** -14, 65504.0)), ("bf16", (2.0, -(2.0 ** -80), 2.0 ** 100))):
        for val in values:
            X = torch.zeros((batch, K), dtype=TORCH[x], device="cuda")
            X[batch - 1] = val
            Y = torch.empty((batch, N), device="cuda")
            q.qtea_w4_gemm_lowbatch(m, X, Y)
            want = torch.zeros((batch, N), device="cuda")
            for n, (k, w) in at.items():
                want[batch - 1, n] = w * val
            assert torch.equal(Y, want), (x, val)


@pytest.mark.parametrize("batch", [1, 16, 40])
def test_the_same_every_time_and_in_a_graph(batch):
    """Random values: the same bits again, on a stream of its own and replayed."""
    for N, K in ((5123, 8224), (10243, 2600), (28675, 1056)):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(N + batch)
        m = q.pack_matrix_w4(torch.randn((N, K), generator=gen, device="cuda"))
        X = torch.randn((batch, K), generator=gen, device="cuda").half()
        Y, Z = torch.empty((batch, N), device="cuda"), torch.empty((batch, N), device="cuda")
        q.qtea_w4_gemm_lowbatch(m, X, Y)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            q.qtea_w4_gemm_lowbatch(m, X, Z)
        for _ in range(3):
            Z.fill_(7)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(Y, Z)
            X.copy_(torch.randn(X.shape, generator=gen, device="cuda"))
            q.qtea_w4_gemm_lowbatch(m, X, Y)
