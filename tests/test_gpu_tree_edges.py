"""Edges of a speculative step's operators on the GPU."""
import decimal
import math
from decimal import Decimal as D

import numpy as np
import pytest
import torch

import paper_2607_16213_gb300 as S
from paper_2607_16213_gb300 import api
import tree_ref as R
from test_gpu_tree import Case, HALF_STEP, check_verify, dev, host, probabilities, run_verify
from test_tree_numbers import PLANS, exact_turns

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_16213_gb300 import build as b
    b.build()
    S.library()


# ---- rotary positions ---------------------------------------------------------------------------
@pytest.mark.parametrize("kw", PLANS, ids=lambda k: "-".join(str(v) for v in k.values()))
def test_rotary_at_far_positions(kw):
    """Angles from the formula in 80 digits: what the 64-bit formula's own angle is off by does not count here.  fp32: sine and
    cosine to 2^-21 as in test_gpu_tree.check_rope."""
    pos = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, -987654321, 2 ** 24 + 1, 1, 0], dtype=np.int64)
    T, d, rot = len(pos), 128, kw["rot"]
    shape = api.make_shape("fp32", 1, 2, 1, d, 8, 64, 64)
    plan = api.rotary_plan(rot, kw["theta"], **{k: v for k, v in kw.items() if k not in ("rot", "theta")})
    x = np.random.default_rng(rot).normal(size=(1, 2, T, d)).astype(np.float32)
    got = host(api.rotary(shape, plan, dev(pos[None], torch.int32), q=dev(x))[0])
    with decimal.localcontext() as c:
        c.prec = 80
        turn = np.array([[float(int(p) * t % 1) for t in exact_turns(**kw)] for p in pos])
    z = plan.amplitude * np.exp(2j * math.pi * turn)
    w = (x[..., :rot // 2] + 1j * x[..., rot // 2:rot].astype(np.float64)) * z
    size = plan.amplitude * (np.abs(x[..., :rot // 2]) + np.abs(x[..., rot // 2:rot]))
    for part, want in ((got[..., :rot // 2], w.real), (got[..., rot // 2:rot], w.imag)):
        err, tol = np.abs(part - want), HALF_STEP["fp32"] * np.abs(want) * 1.01 + size * 2.0 ** -21
        assert (err <= tol).all(), float((err / tol).max())
    np.testing.assert_array_equal(got[..., rot:], x[..., rot:])


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
