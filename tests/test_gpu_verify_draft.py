"""qtea_verify_draft against the oracle's whole numbers: equal decisions."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.serving as sv
import paper_2609_00224_amd as q
from tests.serving_cases import TORCH

pytestmark = pytest.mark.gpu


def _softmax(x):
    e = np.exp(x - x.max(-1, keepdims=True))
    return e / e.sum(-1, keepdims=True)


def _inputs(rng, drafts, vocab, kind, near=0.5):
    """Host inputs of a batch with the given drafts per sequence."""
    n = sum(drafts)
    logits = 3 * rng.standard_normal((n + len(drafts), vocab))
    keep = np.concatenate([np.r_[np.ones(k, bool), False] for k in drafts])
    target = _softmax(logits)
    draft = _softmax(logits[keep] + near * rng.standard_normal((n, vocab)))
    as_type = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(TORCH[kind])  # noqa: E731
    tokens = np.array([rng.choice(vocab, p=d) for d in draft], np.int32).reshape(n)
    u = lambda m: torch.from_numpy(rng.random(m).astype(np.float32))  # noqa: E731
    starts = np.concatenate([[0], np.cumsum([k + 1 for k in drafts])]).astype(np.int32)
    return dict(target=as_type(target), draft=as_type(draft), tokens=torch.from_numpy(tokens), q_start=torch.from_numpy(starts),
                u_accept=u(n), u_sample=u(len(drafts)), drafts=list(drafts))


def _run(x, width, ws=None, pad=0):
    dev = {k: v.cuda() for k, v in x.items() if isinstance(v, torch.Tensor)}
    for name in ("target", "draft"):
        if pad and name in dev:  # rows a stride apart that is no multiple of anything
            wide = torch.full((dev[name].shape[0], dev[name].shape[1] + pad), 0.5, dtype=dev[name].dtype, device="cuda")
            wide[:, :dev[name].shape[1]] = dev[name]
            dev[name] = wide[:, :dev[name].shape[1]]
    n = len(x["q_start"]) - 1
    acc = torch.full((n,), 99, dtype=torch.int32, device="cuda")
    out = torch.full((n, width + 1), 99, dtype=torch.int32, device="cuda")
    q.qtea_verify_draft(dev["target"], dev.get("draft"), dev["tokens"], dev["q_start"], dev["u_accept"], dev["u_sample"], acc, out,
                        q.new_verify_workspace(n) if ws is None else ws)
    return acc.cpu().numpy(), out.cpu().numpy()


def _want(x, width):
    acc, out, at = [], [], 0
    for s, k in enumerate(x["drafts"]):
        t0, n = int(x["q_start"][s]), min(k, width)
        d = x["draft"][at:at + n].double().numpy() if "draft" in x else None
        tok = x["tokens"][at:at + n].numpy()
        a, nxt = sv.verify(x["target"][t0:t0 + n + 1].double().numpy(), d, tok, x["u_accept"][at:at + n].numpy(), x["u_sample"][s].item())
        acc.append(a)
        out.append(list(tok[:a]) + [nxt] + [-1] * (width - a))
        at += k
    return np.array(acc), np.array(out)


def _check(x, width, **more):
    got, want = _run(x, width, **more), _want(x, width)
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("drafts,vocab", [([1], 1), ([2], 7), ([4], 1000), ([0], 33), ([3, 0, 5, 1], 2049), ([2] * 70, 65),
                                          ([7, 6], 5003), ([1, 2], 40000), ([80, 3], 50)])
def test_decisions_are_the_oracles(drafts, vocab, kind):
    rng = np.random.default_rng([len(drafts), vocab, len(kind)])
    x = _inputs(rng, drafts, vocab, kind)
    _check(x, max(drafts))
    _check(x, max(drafts), pad=3)
    del x["draft"]  # deterministic drafts
    _check(x, max(drafts))


def test_a_batch_smaller_than_the_drafts_ignores_the_rest():
    x = _inputs(np.random.default_rng(1), [5, 2, 6], 300, "f32", near=0.01)
    for width in (0, 1, 3, 9):
        _check(x, width)


def test_edges_of_the_random_numbers():
    """0 accepts whatever the target can emit, the largest samples the last token with mass."""
    rng = np.random.default_rng(2)
    for u in (0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, float("nan")):
        x = _inputs(rng, [3, 2], 400, "f32")
        x["u_accept"].fill_(u)
        x["u_sample"].fill_(u)
        x["target"][:, 350:] = 0
        x["target"][:, :9] = 0
        got = _run(x, 3)
        for name in ("u_accept", "u_sample"):  # the definition's limits
            x[name] = torch.full_like(x[name], min(max(u, 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0)
        want = _want(x, 3)
        np.testing.assert_array_equal(got[0], want[0])
        np.testing.assert_array_equal(got[1], want[1])


def test_degenerate_rows():
    """Equal distributions (nothing left after a forced rejection), one-hot
    targets, rows without mass, values that are no probabilities, tokens
    outside the vocabulary."""
    rng = np.random.default_rng(3)
    x = _inputs(rng, [2, 2, 2, 2, 2, 1], 100, "f32")
    t, d = x["target"], x["draft"]
    d[0:2] = t[0:2]                                     # p = q: always accepted
    t[3:5], d[2:4] = 0.0, 0.01
    t[3, 17] = t[4, 99] = 1.0                           # one-hot target: the first rejection emits its token
    t[6:9] = 0.0                                        # no mass: -1
    t[9, :50], t[9, 50:] = float("nan"), 0.02           # NaN counts as 0
    d[6] = 0.0
    t[12], t[12, 5] = -1.0, 7.0                         # limited to [0, 1]
    x["tokens"][8] = 100
    x["tokens"][10] = -1
    _check(x, 2)
    t[15:17] = d[10:11]                                 # equal rows and a token outside: the target's own row
    _check(x, 2)


def test_sequences_without_rows():
    x = _inputs(np.random.default_rng(4), [2, 1], 60, "f32")
    x["q_start"] = torch.tensor([0, 0, 3, 3, 5, 5], dtype=torch.int32)
    x["u_sample"] = torch.rand(5)
    acc, out = _run(x, 2)
    y = dict(x, q_start=torch.tensor([0, 3, 5], dtype=torch.int32), u_sample=x["u_sample"][[1, 3]])
    want = _want(y, 2)
    assert list(acc[[0, 2, 4]]) == [0, 0, 0] and (out[[0, 2, 4]] == -1).all()
    np.testing.assert_array_equal(acc[[1, 3]], want[0])
    np.testing.assert_array_equal(out[[1, 3]], want[1])


def test_sampled_tokens_follow_the_target():
    """Drafts from q, verified: the first emitted token is distributed as p
    (4000 sequences, 12 tokens; a chi-square far past its 1e-6 point fails)."""
    rng = np.random.default_rng(5)
    n, vocab = 4000, 12
    p, d = _softmax(rng.standard_normal(vocab)), _softmax(rng.standard_normal(vocab))
    x = dict(target=torch.from_numpy(np.tile(p, (2 * n, 1))).float(), draft=torch.from_numpy(np.tile(d, (n, 1))).float(),
             tokens=torch.from_numpy(rng.choice(vocab, n, p=d).astype(np.int32)), q_start=torch.arange(0, 2 * n + 1, 2, dtype=torch.int32),
             u_accept=torch.from_numpy(rng.random(n).astype(np.float32)), u_sample=torch.from_numpy(rng.random(n).astype(np.float32)))
    _, out = _run(x, 1)
    seen = np.bincount(out[:, 0], minlength=vocab)
    chi2 = ((seen - n * p) ** 2 / (n * p)).sum()
    assert chi2 < 50  # 11 degrees of freedom: 1e-6 lies at 49


def test_a_workspace_and_a_graph_serve_call_after_call():
    rng = np.random.default_rng(6)
    x = _inputs(rng, [3, 4, 0], 9001, "f32")
    ws = q.new_verify_workspace(3)
    dev = {k: v.cuda() for k, v in x.items() if isinstance(v, torch.Tensor)}
    acc, out = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty((3, 5), dtype=torch.int32, device="cuda")
    call = lambda: q.qtea_verify_draft(dev["target"], dev["draft"], dev["tokens"], dev["q_start"], dev["u_accept"], dev["u_sample"], acc, out, ws)  # noqa: E731
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        call()
    for i in range(5):
        for name in ("u_accept", "u_sample"):
            x[name] = torch.from_numpy(rng.random(len(x[name])).astype(np.float32))
            dev[name].copy_(x[name])
        want = _want(x, 4)
        for run in (g.replay, call):
            acc.fill_(99)
            out.fill_(99)
            run()
            torch.cuda.synchronize()
            np.testing.assert_array_equal(acc.cpu().numpy(), want[0])
            np.testing.assert_array_equal(out.cpu().numpy(), want[1])
