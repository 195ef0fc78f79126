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
