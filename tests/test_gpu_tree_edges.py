"""Edges of a speculative step's operators on the GPU."""
import decimal
import math
from decimal import Decimal as D
from fractions import Fraction

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


def left_of(p, q, tokens):
    """The weights after the rejection of each of `tokens` in turn, without error."""
    P = [int(x * 2.0 ** 160) for x in p.astype(np.float64)]
    if q is None:
        for x in tokens:
            P[x] = 0
        return [Fraction(x, 2 ** 160) for x in P]
    Q = [int(x * 2.0 ** 160) for x in q.astype(np.float64)]
    A, r = Fraction(0), [Fraction(x, 2 ** 160) for x in P]
    M = Fraction(1)
    for _ in tokens:
        A += M
        num, den = A.numerator, A.denominator
        whole = [max(a * den - num * b, 0) for a, b in zip(P, Q)]
        M = Fraction(sum(whole), den * 2 ** 160)
        r = [Fraction(x, den * 2 ** 160) for x in whole]
    return r


def bring_border(p, q, tokens, u0, k, sign):
    """Adds to entries 0 to 2 (without weight in q, each finer than the one before) until the running sum of some entry lies 1 to 2
    times the documented distance, 2^-42 (1 + k / mass left) of the whole, from u0 of the whole, above it or below (`sign`).
    Returns the token that u0 draws."""
    for step in range(24):
        r = left_of(p, q, tokens)
        Z = sum(r)
        at, c, j, below = Fraction(float(u0)) * Z, Fraction(0), 0, Fraction(0)
        away = Fraction(2) ** -42 * (Z + k) * Fraction(3, 2)
        for i, x in enumerate(r):  # the last border that is not far above
            c += x
            if c - at > 4 * away:
                break
            if x > 0:
                j, below = i, c
        gap = sign * away - (below - at)
        if abs(gap) < away / 3:
            return j if sign > 0 else next(i for i in range(j + 1, len(r)) if r[i] > 0)
        knob = min(2, step // 6)
        move = float(gap / (1 - Fraction(float(u0))))
        p[knob] = np.float32(float(p[knob]) + (move if knob == 2 else 0.9 * max(0.0, move)))  # (the rest is left to the finer ones)
        assert p[knob] >= 0
    raise AssertionError("the border was not brought there")


@pytest.mark.parametrize("drawn,k", [(True, 0), (True, 1), (True, 2), (True, 3), (False, 2)])
@pytest.mark.parametrize("V,eps", [(2000, 0.3), (8192, 0.01), (8191, 0.0005)])
def test_tree_verify_draws_near_a_border(drawn, k, V, eps):
    """A draft that is close to its target leaves little mass: borders between tokens are right to 2^-42 (1 + k / mass) of it."""
    rng = np.random.default_rng(V + k)
    cases = []
    for u0, sign in ((0.5, 1), (0.5, -1), (0.75, 1), (0.2501, -1)):
        q = 0.5 + rng.random(V)
        p = np.abs(q * (1 + eps * rng.normal(size=V)))
        p, q = (p / p.sum()).astype(np.float32), (q / q.sum()).astype(np.float32)
        q[:3] = 0
        p[:3] = 0
        tokens = [int(x) for x in np.argsort(p[3:] / q[3:])[:k] + 3]
        u0 = np.float32(u0)
        want = bring_border(p, q if drawn else None, tokens, u0, k if drawn else 0, sign)
        cases.append((p, q, tokens, u0, want))
    T = k + 1
    target, draft = (np.stack([np.stack([c[i]] * T) for c in cases]) for i in (0, 1))
    tok = np.array([[0] + c[2] for c in cases])
    u = np.full((len(cases), T), 1 - 2.0 ** -24, dtype=np.float32)
    u[:, 0] = [c[3] for c in cases]
    got = run_verify(tok, np.array([[-1] + [0] * k] * len(cases)), u, target, draft if drawn else None)
    assert list(got[0]) == [1] * len(cases)
    assert list(got[2]) == [c[4] for c in cases]


@pytest.mark.parametrize("V", [2, 300, 5000])
def test_tree_verify_rows_that_are_left_without_mass(V):
    """Picked drafts that are all that a row holds, each rejected: the row's sum is a rounding below 1, so nothing is wrong with it
    and the last token follows.  A row that never had mass is reported."""
    p = np.zeros((1, 3, V), dtype=np.float32)
    p[:, :, 0], p[:, :, 1] = 0.3, np.float32(0.7) - np.float32(2.0 ** -22)
    tokens, parents = np.array([[0, 0, 1]]), np.array([[-1, 0, 0]])
    u = np.array([[0.5, 0.999, 1 - 2.0 ** -24]], dtype=np.float32)
    ws = api.Workspace(256)
    got = run_verify(tokens, parents, u, p, None, None, ws)
    check_verify(got, tokens, parents, u, p, None)
    assert got[2][0] == V - 1 and ws.errors() == 0
    for draft in (None, p):
        got = run_verify(tokens, parents, u, np.zeros_like(p), draft, None, ws)
        assert got[0][0] == 1 and got[2][0] == V - 1 and ws.errors() == S.SELKV_DEVERR_VALUE
    # a row without mass that the walk leaves by a child is not drawn from
    q = p.copy()
    q[0, 0] = 0
    q[0, 0, 1] = 1.0
    q[0, 1] = 0
    got = run_verify(tokens, np.array([[-1, 0, 0]]), u, q, None, None, ws)
    assert list(got[1][0]) == [0, 2, -1] and ws.errors() == 0


# ---- attention ----------------------------------------------------------------------------------
@pytest.mark.parametrize("hkv,d,cap,lengths,T,counts", [
    (1, 128, 300, [300], 65, None), (2, 128, 700, [613, 1], 128, [128, 97]), (4, 64, 90, [64, 0, 90], 100, [100, 66, 64]),
    (8, 64, 3000, [2999], 127, None), (2, 128, 64, [0, 0], 65, [65, 65]), (3, 128, 130, [128, 129, 17], 128, [1, 64, 128])])
@pytest.mark.parametrize("bias,parents", [("ratio", "tree"), (None, "chain"), ("masked", "forest")])
def test_tree_attn_one_query_head_and_two_tiles_of_tokens(hkv, d, cap, lengths, T, counts, bias, parents):
    """bf16, a query head a KV head, 65 to 128 tokens: all rows in one accumulator, and the tokens' own rows in two tiles, which
    the two chains take each one of or, where they lie in different pieces, one after the other."""
    c = Case("bf16", len(lengths), hkv, hkv, d, cap, lengths, T, counts, bias=bias, parents=parents)
    before = torch.full_like(c.q, 7.0)
    ws = api.Workspace(S.selkv_tree_attn_workspace_size(c.shape, T))
    out = c.run(out=before.clone(), workspace=ws)
    c.check(out, before=before)
    assert ws.errors() == 0
    assert torch.equal(c.run(out=before.clone(), workspace=ws), out)


@pytest.mark.parametrize("hq,hkv,T,cap", [(16, 2, 20, 137), (8, 1, 40, 600), (4, 1, 70, 64), (2, 1, 100, 200), (1, 1, 90, 2000), (8, 2, 96, 30)])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_tree_attn_values_that_are_no_numbers(hq, hkv, T, cap, what):
    """bf16 with more than 128 query rows, where both accumulators' warps clear the same drafted values that are no numbers, and with
    two tiles of tokens: such a value reaches the tokens that see it, in its element alone."""
    for seed in range(4):
        c = Case("bf16", 2, hq, hkv, 64, cap, [cap, cap // 2], T, None, seed=seed, parents="forest")
        clean = c.run()
        rng = np.random.default_rng(seed)
        sees = [R.ancestors(c.pr[b], T) for b in range(2)]
        hit = np.zeros((2, hkv, T, 64), dtype=bool)
        for _ in range(5):
            b, kv, t, e = int(rng.integers(2)), int(rng.integers(hkv)), int(rng.integers(T)), int(rng.integers(64))
            c.v[b, kv, t, e] = what
            hit[b, kv, :, e] |= sees[b][:, t]
        hit = torch.as_tensor(np.repeat(hit, hq // hkv, axis=1)).cuda()
        got = c.run()
        assert torch.equal(got[~hit], clean[~hit])
        bad = got[hit].float()
        assert bool((bad.isnan() if math.isnan(what) else bad == what).all())


# ---- offsets past 32 bits -----------------------------------------------------------------------
def test_rotary_rows_past_32_bits():
    """A prompt whose last rows begin past 2^31 elements: to the bit what a call over those rows alone gives."""
    T, n = 2 ** 24 + 1001, 900
    shape, plan = api.make_shape("bf16", 1, 1, 1, 128, 8, 64, 64), api.rotary_plan(128)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")[None]
    k = torch.zeros((1, 1, T, 128), dtype=torch.bfloat16, device="cuda")
    k[:, :, -n:] = torch.randn((1, 1, n, 128), generator=torch.Generator("cuda").manual_seed(1), device="cuda").bfloat16()
    want = api.rotary(shape, plan, pos[:, -n:].contiguous(), k=k[:, :, -n:].contiguous())[1]
    api.rotary(shape, plan, pos, k=k, out=(None, k))
    assert torch.equal(k[:, :, -n:], want) and not k[:, :, :-n].any()


@pytest.mark.parametrize("drawn", [True, False])
def test_tree_verify_rows_past_32_bits(drawn):
    """1024 sequences of the largest vocabulary: the last ones' rows begin past 2^31 entries."""
    B, T, V = 1024, 3, 1 << 20
    rng = np.random.default_rng(2)
    target = torch.zeros((B, T, V), device="cuda")
    draft = torch.zeros((B, T, V), device="cuda") if drawn else None
    at = rng.integers(0, V, size=(B, T, 4))
    p, q = (np.tile(np.array(x, dtype=np.float32) / 16, (B, T, 1)) for x in ((8, 4, 3, 1), (2, 2, 6, 6)))
    for b in range(B):
        for t in range(T):
            at[b, t] = np.sort(rng.choice(V, 4, replace=False))
    rows = torch.as_tensor(at).cuda()
    target.scatter_(2, rows, dev(p))
    if drawn:
        draft.scatter_(2, rows, dev(q))
    tokens = np.zeros((B, T), dtype=np.int32)
    tokens[:, 1], tokens[:, 2] = at[np.arange(B), 0, rng.integers(0, 4, B)], at[np.arange(B), 1, rng.integers(0, 4, B)]
    u = np.minimum(rng.random((B, T)).astype(np.float32), np.float32(1 - 2.0 ** -24))
    ws = api.Workspace(256)
    got = [x.cpu().numpy() for x in api.tree_verify(dev(tokens, torch.int32), None, dev(u), target, draft, workspace=ws)]
    assert ws.errors() == 0
    del target, draft
    # the same over the entries that have weight
    for b in list(range(0, 1024, 41)) + [1021, 1022, 1023]:
        # tokens as their places in the four of their parent's row
        of = [0] + [int(np.where(at[b, t - 1] == tokens[b, t])[0][0]) for t in (1, 2)]
        a, path, nxt = R.tree_verify(of, [-1, 0, 1], u[b].astype(np.float64), p[b].astype(np.float64), q[b].astype(np.float64) if drawn else None, T)
        assert got[0][b] == a and list(got[1][b]) == path + [-1] * (T - a) and got[2][b] == at[b, path[-1], nxt]
