"""The operators of a speculative step on the host: their plain forms against closed forms, the rotary plan, and
the refusals (no call here reaches a launch)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2607_16213_gb300 as S
from paper_2607_16213_gb300 import api
import tree_ref as R

FAKE = 1 << 40
INV, UNS, WS = S.SELKV_ERR_INVALID_ARG, S.SELKV_ERR_UNSUPPORTED, S.SELKV_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2607_16213_gb300 import build as b
    b.build()
    return S.library()


# ---- the plain forms ----------------------------------------------------------------------------
def test_tree_attn_of_equal_keys_is_the_mean_of_what_is_seen():
    rng = np.random.default_rng(0)
    parents = np.array([-1, 0, 0, 2, -1])
    v = rng.normal(size=(1, 5, 8))
    K, V = np.zeros((1, 3, 8)), rng.normal(size=(1, 3, 8))
    out, _, _ = R.tree_attn(rng.normal(size=(2, 5, 8)), K, V, None, 3, np.zeros((1, 5, 8)), v, parents, 5)
    seen = [[0], [0, 1], [0, 2], [0, 2, 3], [4]]
    for t, s in enumerate(seen):
        want = np.concatenate([V[0], v[0, s]]).mean(0)
        np.testing.assert_allclose(out[:, t], np.stack([want, want]), rtol=0, atol=1e-14)


@pytest.mark.parametrize("drawn", [True, False])
def test_verification_leaves_the_targets_distribution(drawn):
    """Chance enters through the numbers alone: over a grid of them the next token (the accepted child or the one drawn)
    has the target's distribution, up to the grid's step."""
    p = np.array([0.05, 0.45, 0.3, 0.2])
    q = np.array([0.4, 0.1, 0.3, 0.2])
    target = np.stack([p] * 3)
    draft = np.stack([q] * 3) if drawn else None
    got = np.zeros(4)
    n = 24
    grid = (np.arange(n) + 0.5) / n
    pairs = [(x, y, q[x] * q[y]) for x in range(4) for y in range(4)] if drawn else [(0, 1, 1.0)]
    for x, y, w in pairs:
        for u1 in grid:
            for u2 in grid:
                for u0 in grid:
                    a, path, nxt = R.tree_verify([0, x, y], [-1, 0, 0], [u0, u1, u2], target, draft, 3)
                    got[nxt if a == 1 else (x, y)[path[1] - 1]] += w / n ** 3
    np.testing.assert_allclose(got, p, atol=2.0 / n)


# ---- the rotary plan ----------------------------------------------------------------------------
@pytest.mark.parametrize("kw", [
    dict(rot=128, theta=1e4), dict(rot=64, theta=5e5), dict(rot=2, theta=1e4), dict(rot=18, theta=0.5),
    dict(rot=128, theta=1e4, scaling="linear", factor=4.0),
    dict(rot=128, theta=5e5, scaling="wavelength", factor=8.0, original=8192, low=1.0, high=4.0),
    dict(rot=64, theta=1e4, scaling="ramp", factor=16.0, original=4096, low=1.0, high=32.0),
    dict(rot=32, theta=10.0, scaling="ramp", factor=2.0, original=64, low=1.0, high=1e6),
])
def test_rotary_plan_is_the_formula(kw):
    plan = api.rotary_plan(kw["rot"], kw["theta"], **{k: v for k, v in kw.items() if k not in ("rot", "theta")})
    want = R.frequencies(**kw) / (2 * math.pi)
    want -= np.floor(want)
    got = np.array([float(plan.turns[f]) / 2.0 ** 64 for f in range(kw["rot"] // 2)])
    # pow and log of 64 bits on both sides: a few last places of the frequency (turns a position below 1)
    np.testing.assert_allclose(got, want, rtol=0, atol=2.0 ** -50)
    assert all(plan.turns[f] == 0 for f in range(kw["rot"] // 2, 64))
    want = 0.1 * math.log(kw["factor"]) + 1.0 if kw.get("scaling") == "ramp" else 1.0
    assert plan.amplitude == np.float32(want)


def test_rotary_plan_refusals():
    for args in ((0,), (1,), (3,), (130,), (-2,)):
        with pytest.raises(S.SelKVError):
            api.rotary_plan(*args)
    for kw in (dict(theta=0.0), dict(theta=-1.0), dict(theta=math.inf), dict(theta=math.nan), dict(layout="rows"),
               dict(scaling="other"), dict(scaling="linear", factor=0.0), dict(scaling="linear", factor=math.nan),
               dict(scaling="wavelength", factor=2.0), dict(scaling="ramp", factor=2.0, original=64, low=0.0),
               dict(scaling="wavelength", factor=2.0, original=64, low=4.0, high=4.0),
               dict(scaling="ramp", factor=2.0, original=64, theta=1.0), dict(amplitude=-1.0), dict(amplitude=math.inf)):
        with pytest.raises(S.SelKVError) as e:
            api.rotary_plan(64, **kw)
        assert e.value.status == INV
    assert S.selkv_rotary_init(S.selkv_rotary(), 64, 0, 1e4) == INV
    assert S.library().selkv_rotary_init(None, 64, 1, 1e4, None) == INV


# ---- refusals -----------------------------------------------------------------------------------
def shape(**kw):
    base = dict(dtype=S.SELKV_BF16, batch=2, num_q_heads=32, num_kv_heads=8, head_dim=128, obs_window=64, n_cap=4096,
                m_cap=4160)
    base.update(kw)
    return S.selkv_shape(**base)


def rotary(s=None, plan=None, T=5, pos=FAKE, q=FAKE, k=FAKE, qo=FAKE, ko=FAKE):
    return S.selkv_rotary_apply(s or shape(), plan if plan is not None else api.rotary_plan(64), T, pos, q, k, qo, ko, 0, 0)


def attn(s=None, T=5, parents=None, counts=None, q=FAKE, K=FAKE, V=FAKE, bias=None, lengths=FAKE, k=FAKE, v=FAKE, out=FAKE,
         ws=FAKE, wsb=1 << 40):
    return S.selkv_tree_attn(s or shape(), T, parents, counts, q, K, V, bias, lengths, k, v, out, ws, wsb, 0)


def verify(batch=2, T=5, parents=None, counts=None, vocab=100, tokens=FAKE, uniforms=FAKE, target=FAKE, draft=None,
           accepted=FAKE, path=FAKE, nxt=FAKE, ws=FAKE, wsb=1 << 40):
    return S.selkv_tree_verify(batch, T, parents, counts, vocab, tokens, uniforms, target, draft, accepted, path, nxt, ws, wsb, 0)


def commit(s=None, T=5, path=FAKE, accepted=FAKE, ws=FAKE, wsb=1 << 40, layers=2, **kw):
    step = 1 << 30
    cols = {n: [FAKE + (i * 7 + j) * step for j in range(layers)] for i, n in enumerate(("kn", "vn", "K", "V", "bias", "len"))}
    cols.update(kw)
    return S.selkv_tree_commit(s or shape(), T, path, accepted, cols["kn"], cols["vn"], cols["K"], cols["V"], cols["bias"],
                               cols["len"], ws, wsb, 0)


@pytest.mark.parametrize("call", [rotary, attn, commit])
def test_shape_refusals(call):
    for kw in (dict(dtype=2), dict(batch=0), dict(batch=1025), dict(num_kv_heads=7), dict(num_kv_heads=33, num_q_heads=33),
               dict(num_q_heads=0), dict(num_q_heads=17, num_kv_heads=1)):
        assert call(s=shape(**kw)) == INV, kw
    for d in (32, 96, 256):
        assert call(s=shape(head_dim=d)) == UNS


def test_rotary_refusals():
    for kw in (dict(T=0), dict(T=-1), dict(pos=0), dict(pos=FAKE + 2), dict(q=None), dict(qo=None), dict(k=None), dict(ko=None),
               dict(q=None, qo=None, k=None, ko=None), dict(q=FAKE + 8), dict(k=FAKE + 2), dict(qo=FAKE + 4), dict(ko=FAKE + 8),
               dict(plan=S.selkv_rotary()), dict(plan=api.rotary_plan(128), s=shape(head_dim=64))):
        assert rotary(**kw) == INV, kw
    assert S.library().selkv_rotary_apply(ctypes.byref(shape()), None, 5, FAKE, FAKE, FAKE, FAKE, FAKE, 0, 0) == INV


def test_tree_attn_refusals():
    for kw in (dict(T=0), dict(T=129), dict(T=-3), dict(q=0), dict(K=0), dict(V=0), dict(lengths=0), dict(k=0), dict(v=0),
               dict(out=0), dict(q=FAKE + 8), dict(K=FAKE + 2), dict(V=FAKE + 4), dict(lengths=FAKE + 4), dict(k=FAKE + 8),
               dict(v=FAKE + 8), dict(out=FAKE + 2), dict(bias=FAKE + 4), dict(parents=FAKE + 2), dict(counts=FAKE + 1),
               dict(s=shape(m_cap=0))):
        assert attn(**kw) == INV, kw
    assert attn(s=shape(batch=1024, m_cap=1 << 18)) == UNS
    need = S.selkv_tree_attn_workspace_size(shape(), 5)
    assert need > 256
    for kw in (dict(ws=0), dict(ws=FAKE + 16), dict(wsb=need - 1)):
        assert attn(**kw) == WS, kw
    for s, T in ((shape(head_dim=96), 5), (shape(m_cap=0), 5), (shape(batch=0), 5), (shape(), 0), (shape(), 129),
                 (shape(batch=1024, m_cap=1 << 18), 5)):
        assert S.selkv_tree_attn_workspace_size(s, T) == 0


def test_tree_verify_refusals():
    for kw in (dict(batch=0), dict(batch=1025), dict(T=0), dict(T=129), dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(tokens=0),
               dict(uniforms=0), dict(target=0), dict(accepted=0), dict(path=0), dict(nxt=0), dict(tokens=FAKE + 2),
               dict(target=FAKE + 4), dict(draft=FAKE + 8), dict(parents=FAKE + 2), dict(counts=FAKE + 2), dict(nxt=FAKE + 1)):
        assert verify(**kw) == INV, kw
    for kw in (dict(ws=0), dict(ws=FAKE + 16), dict(wsb=255)):
        assert verify(**kw) == WS, kw
    assert S.selkv_tree_verify_workspace_size(2, 5, 100) >= 256
    for args in ((0, 5, 100), (1025, 5, 100), (2, 0, 100), (2, 129, 100), (2, 5, 0), (2, 5, (1 << 20) + 1)):
        assert S.selkv_tree_verify_workspace_size(*args) == 0


def test_tree_commit_refusals():
    two = [FAKE, FAKE + (1 << 30)]
    for kw in (dict(T=0), dict(T=129), dict(path=0), dict(path=FAKE + 2), dict(accepted=0), dict(accepted=FAKE + 1),
               dict(layers=0), dict(layers=129), dict(kn=[FAKE, 0]), dict(vn=[0, FAKE]), dict(K=[FAKE, FAKE + 8]),
               dict(V=[FAKE + 2, FAKE]), dict(len=[FAKE, 0]), dict(len=[FAKE + 4, FAKE]), dict(bias=[FAKE + 4, None]),
               dict(len=[FAKE, FAKE]), dict(K=[FAKE, FAKE]), dict(V=[FAKE, FAKE]), dict(s=shape(m_cap=0)), dict(kn=two[:1])):
        assert commit(**kw) == INV, kw
    for kw in (dict(ws=0), dict(ws=FAKE + 16), dict(wsb=255)):
        assert commit(**kw) == WS, kw
    assert S.selkv_tree_commit_workspace_size(shape()) >= 256
    assert S.selkv_tree_commit_workspace_size(shape(batch=0)) == 0


def test_helpers_refuse_host_tensors():
    s = api.make_shape("bf16", 1, 4, 2, 64, 8, 64, 64)
    z = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16)
    cache = api.CompressedCache(s, z, z, None, torch.zeros(1, dtype=torch.int32))
    ints = torch.zeros((1, 2), dtype=torch.int32)
    for call in (lambda: api.rotary(s, api.rotary_plan(64), ints, q=z), lambda: api.tree_attn(cache, z, z, z),
                 lambda: api.tree_verify(ints, None, torch.zeros(1, 2), torch.zeros(1, 2, 9)),
                 lambda: api.tree_commit(cache, z, z, ints, ints[0])):
        with pytest.raises(S.SelKVError) as e:
            call()
        assert e.value.status == INV
