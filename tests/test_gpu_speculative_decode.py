"""The serving operators together: examples/speculative_decode.py."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROMPTS = [[1, 2, 3, 4, 5], [6, 7], [8, 9, 10, 11]]


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("speculative_decode", os.path.join(ROOT, "examples", "speculative_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("fmt", ["f16", "e4m3", "e2m1"])
def test_greedy_tokens_do_not_depend_on_the_drafts(example, fmt):
    """With all of the target's mass on one token, verified drafts change how
    many steps the tokens take and not the tokens."""
    plain = example.generate(fmt, PROMPTS, 12, 0, 0)
    drafted = example.generate(fmt, PROMPTS, 12, 3, 0)
    for a, b, p in zip(plain, drafted, PROMPTS):
        assert len(a) == len(p) + 12 and len(b) >= len(a)
        assert b[:len(a)] == a


def test_a_step_is_attention_over_what_was_cached(example):
    """The same tokens in one pass or one by one: the same distributions."""
    model = [example.Decoder("f16", 1, 40, seed=3) for _ in range(2)]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    tokens = [5, 17, 3, 99, 100, 640, 2, 8]
    whole = model[0].probabilities(i32(tokens), i32([0, len(tokens)]), i32([len(tokens)]), 1.0)
    for k, t in enumerate(tokens):
        one = model[1].probabilities(i32([t]), i32([0, 1]), i32([k + 1]), 1.0)
        assert torch.allclose(one[0], whole[k], rtol=2e-2, atol=1e-5)


def test_sampling_runs(example):
    got = example.generate("e4m3", PROMPTS, 6, 3, 1.0)
    for g, p in zip(got, PROMPTS):
        assert len(p) + 6 <= len(g) <= len(p) + 24 and all(0 <= t < example.VOCAB for t in g)
