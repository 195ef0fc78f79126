"""The layer operators together with the products, cache and attention:
examples/decode.py against the same model in 64 bits."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

import paper_2609_00224_amd as q

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("decode", os.path.join(ROOT, "examples", "decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _dense(linear):
    """A linear's matrix, fp64."""
    if linear.eight_bits:
        W = torch.empty((linear.N, linear.K), device="cuda")
        q.qtea_w4_unpack(linear.m, W)
        return W.double()
    T, alpha, v, S, R, idx = linear.parts
    W = alpha.double()[:, None] * T.double() * v.double()
    rows = 4 * torch.arange(R.shape[1], device="cuda") + idx.long()  # [nS][N / 4]
    W[rows, S.long()[:, None].expand_as(rows)] += R.double()
    return W


def _reference(ex, model, tokens):
    """The model's logits for one sequence, without a rounding in between."""
    n = len(tokens)
    norm = lambda x, w: x / torch.sqrt((x * x).mean(-1, keepdim=True) + ex.EPS) * w.double()  # noqa: E731
    x = model.embed[tokens.long()].double()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.arange(n, device="cuda").double()[:, None] * model.freq.double())[:, None]
    hidden = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)

    def turned(y):
        z = torch.complex(y[..., :ex.DIM // 2], y[..., ex.DIM // 2:]) * turn
        return torch.cat((z.real, z.imag), -1)

    for norm1, qkv, out, norm2, gate_up, down in model.layers:
        y = (norm(x, norm1) @ _dense(qkv).T).view(n, -1, ex.DIM)
        H, V = ex.HEADS, ex.KV_HEADS
        Q, K, val = turned(y[:, :H]), turned(y[:, H:H + V]), y[:, H + V:]
        rows = []
        for h in range(H):
            g = h // (H // V)
            s = (Q[:, h] @ K[:, g].T) * ex.DIM ** -0.5
            rows.append(torch.softmax(s.masked_fill(hidden, -torch.inf), -1) @ val[:, g])
        x = x + torch.cat(rows, -1) @ _dense(out).T
        y = norm(x, norm2) @ _dense(gate_up).T
        g, u = y[:, :ex.INNER], y[:, ex.INNER:]
        x = x + (g * torch.sigmoid(g) * u) @ _dense(down).T
    return norm(x, model.last) @ _dense(model.head).T


@pytest.mark.parametrize("fmt,first", [("f16", 1), ("f16", 33), ("e4m3", 5)])
def test_the_decoder_computes_its_formula(example, fmt, first):
    """A prompt in one pass and the rest token by token.  Roundings on the way
    to a logit: E4M3 at the norm and the gate of one feed-forward part and before the
    head (2^-4 at most, about 2^-5.8 in the mean of their squares: 3 of them, and
    the keys, values in 8 bits: 4 more), those of fp16 far below.  Errors of
    independent signs: the root of their number, twice that for what the
    scores' exponentials make of it."""
    n = 40
    tokens = torch.randint(0, example.VOCAB, (n,), generator=torch.Generator().manual_seed(3)).int().cuda()
    model = example.Decoder(fmt, 1, n, seed=5)
    got = [model.logits(tokens[:first], _i32([0, first]), _i32([first]))]
    for k in range(first, n):
        got.append(model.logits(tokens[k:k + 1], _i32([0, 1]), _i32([k + 1])))
    got, want = torch.cat(got).double(), _reference(example, model, tokens)
    count = 3 + (4 if fmt == "e4m3" else 0)
    assert (got - want).norm() <= 2 * count ** 0.5 * 2.0 ** -5.8 * want.norm()


@pytest.mark.parametrize("fmt", ["bf16", "e2m1"])
def test_generation_runs(example, fmt):
    got = example.generate(fmt, [[1, 2, 3, 4, 5], [6], [8, 9]], 9)
    assert len(got) == 3 and all(len(g) == 9 and all(0 <= t < example.VOCAB for t in g) for g in got)


def test_a_step_as_a_graph(example):
    """One step of two sequences captured once; lengths and tokens change between replays."""
    model, plain = example.Decoder("e4m3", 2, 40, seed=1), example.Decoder("e4m3", 2, 40, seed=1)
    tokens, start, length = _i32([3, 4]), _i32([0, 1, 2]), _i32([1, 1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        model.logits(tokens, start, length)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        logits = model.logits(tokens, start, length)
    for k in range(6):
        tokens.copy_(_i32([7 * k + 1, 5 * k + 2]))
        length.fill_(k + 1)
        g.replay()
        torch.cuda.synchronize()
        want = plain.logits(tokens, start, length)
        assert torch.equal(logits, want)
