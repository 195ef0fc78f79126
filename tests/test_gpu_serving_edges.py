"""Serving operators at the edges of what their arguments may be."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle.serving as sv
import paper_2609_00224_amd as q
from tests.serving_cases import TORCH, Paged, attention_reference, rounded
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
