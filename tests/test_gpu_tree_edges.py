"""Edges of a speculative step's operators on the GPU."""
import math

import numpy as np
import pytest
import torch

import paper_2607_16213_gb300 as S
from paper_2607_16213_gb300 import api
import tree_ref as R
from test_gpu_tree import Case, check_verify, dev, probabilities, run_verify

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_16213_gb300 import build as b
    b.build()
    S.library()


# ---- verification -------------------------------------------------------------------------------
@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("V", [7, 500, 4096])
def test_tree_verify_takes_negative_zeros_for_zeros(V, drawn):
    """-0 as a probability or a number: what +0 gives, and nothing reported."""
    T = 5
    rng = np.random.default_rng(V)
    parents = np.array([[-1, 0, 0, 0, 3]] * 4)
    tokens = rng.integers(0, V, size=(4, T)).astype(np.int32)
    target, draft = (probabilities(rng, (4, T, V), 1.0) for _ in range(2))
    u = np.full((4, T), 0.999, dtype=np.float32)
    u[:, 0] = [0.0, 0.3, 0.9, 0.0]
    u[1, 3] = 0.0
    for b in range(4):
        target[b, :, tokens[b, 1]] = 0.0  # (a tried child's own, and an entry that a draw passes)
        target[b, :, 0] = 0.0
        draft[b, :, tokens[b, 2]] = 0.0
    ws = api.Workspace(256)
    want = run_verify(tokens, parents, u, target, draft if drawn else None, None, ws)
    check_verify(want, tokens, parents, u, target, draft if drawn else None)
    neg = [np.where(x == 0, np.float32(-0.0), x) for x in (u, target, draft)]
    assert all(np.signbit(x).any() for x in neg)
    got = run_verify(tokens, parents, neg[0], neg[1], neg[2] if drawn else None, None, ws)
    assert all(np.array_equal(x, y) for x, y in zip(got, want))
    assert ws.errors() == 0
