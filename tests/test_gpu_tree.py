"""The operators of a speculative step on the GPU against their plain forms in 64 bits (tree_ref.py)."""
import math

import numpy as np
import pytest
import torch

import paper_2607_16213_gb300 as S
from paper_2607_16213_gb300 import api
import tree_ref as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
LOWEST = -3.4028234663852886e38


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_16213_gb300 import build as b
    b.build()
    S.library()


def dev(x, dtype=None):
    t = torch.as_tensor(np.ascontiguousarray(x))
    return (t if dtype is None else t.to(dtype)).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


# ---- rotary positions ---------------------------------------------------------------------------
ROPES = [
    dict(dtype="bf16", d=128, rot=128, layout="half"),
    dict(dtype="bf16", d=128, rot=128, layout="interleaved"),
    dict(dtype="bf16", d=64, rot=32, layout="half", theta=5e5),
    dict(dtype="bf16", d=128, rot=32, layout="interleaved"),
    dict(dtype="bf16", d=128, rot=6, layout="half"),
    dict(dtype="bf16", d=64, rot=10, layout="interleaved"),
    dict(dtype="fp32", d=64, rot=64, layout="half"),
    dict(dtype="fp32", d=128, rot=24, layout="interleaved"),
    dict(dtype="fp32", d=128, rot=2, layout="interleaved"),
    dict(dtype="fp32", d=64, rot=62, layout="half"),
    dict(dtype="bf16", d=128, rot=128, layout="half", scaling="linear", factor=4.0),
    dict(dtype="bf16", d=128, rot=128, layout="half", theta=5e5, scaling="wavelength", factor=8.0, original=8192, high=4.0),
    dict(dtype="fp32", d=128, rot=64, layout="half", scaling="ramp", factor=16.0, original=4096),
]


def rope_case(c, B, T, hq, hkv, seed=0):
    rng = np.random.default_rng(seed)
    shape = api.make_shape(c["dtype"], B, hq, hkv, c["d"], 8, 64, 64)
    how = {k: c[k] for k in ("theta", "scaling", "factor", "original", "low", "high") if k in c}
    plan = api.rotary_plan(c["rot"], layout=c["layout"], **how)
    freq = R.frequencies(c["rot"], **{"theta": 1e4, **how})
    q, k = (dev(rng.normal(size=(B, h, T, c["d"])), DT[c["dtype"]]) for h in (hq, hkv))
    pos = rng.integers(0, 1000, size=(B, T))
    far = rng.random((B, T))
    pos = np.where(far < 0.3, rng.integers(0, 2 ** 20, size=(B, T)), pos)
    pos = np.where(far > 0.9, rng.integers(-2 ** 31, 2 ** 31, size=(B, T)), pos)
    return shape, plan, freq, q, k, pos.astype(np.int32)


def check_rope(got, x, pos, freq, c, plan, transpose=False):
    """Half a step of the type, and fp32: sine and cosine to about 2^-22 (their angle to 2^-24 of half a turn, 2 units in
    the last place of the functions, the amplitude), two products and a sum.  The formula's own angle is p w in 64
    bits: right to |p w| 2^-52."""
    want = R.rotate(host(x), pos, freq, c["layout"], plan.amplitude, transpose)
    size = np.abs(R.rotate(host(x), pos * 0, freq * 0, c["layout"], plan.amplitude))
    mix = size.copy()
    rot = c["rot"]
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if c["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    mix[..., a] += size[..., b]
    mix[..., b] += size[..., a]
    angle = np.zeros_like(mix)
    angle[..., a] = angle[..., b] = np.abs(pos[:, None].astype(np.float64) * freq) * 2.0 ** -50
    tol = HALF_STEP[c["dtype"]] * np.abs(want) * 1.01 + mix * (2.0 ** -21 + angle)
    err = np.abs(host(got) - want)
    assert (err <= tol).all(), float((err / tol).max())
    np.testing.assert_array_equal(host(got)[..., rot:], host(x)[..., rot:])


@pytest.mark.parametrize("c", ROPES, ids=lambda c: "-".join(str(v) for v in c.values()))
@pytest.mark.parametrize("B,T,hq,hkv", [(1, 1, 4, 2), (2, 37, 6, 3), (3, 16, 16, 1)])
def test_rotary(c, B, T, hq, hkv):
    shape, plan, freq, q, k, pos = rope_case(c, B, T, hq, hkv)
    for transpose in (False, True):
        gq, gk = api.rotary(shape, plan, dev(pos), q, k, transpose=transpose)
        for x, y in ((q, gq), (k, gk)):
            for b in range(B):
                check_rope(y[b:b + 1], x[b:b + 1], pos[b:b + 1].reshape(1, T)[0], freq, c, plan, transpose)
    # in place, and one of the two alone
    q2, k2 = q.clone(), k.clone()
    api.rotary(shape, plan, dev(pos), q2, k2, out=(q2, k2), transpose=True)
    assert torch.equal(q2, gq) and torch.equal(k2, gk)
    only, none = api.rotary(shape, plan, dev(pos), k=k, transpose=True)[::-1]
    assert none is None and torch.equal(only, gk)


def test_rotary_long_prompt():
    c = dict(dtype="bf16", d=128, rot=128, layout="half")
    shape, plan, freq, q, k, _ = rope_case(c, 1, 5001, 8, 2)
    pos = np.arange(95000, 100001, dtype=np.int32)
    gq, gk = api.rotary(shape, plan, dev(pos[None]), q, k)
    check_rope(gq, q, pos, freq, c, plan)
    check_rope(gk, k, pos, freq, c, plan)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_gradient(layout):
    """The transpose is the gradient: against the formula's differences (the operator is linear, so a difference of any
    size is exact up to rounding)."""
    c = dict(dtype="fp32", d=64, rot=48, layout=layout)
    shape, plan, freq, q, _, pos = rope_case(c, 1, 3, 1, 1)
    pos = np.abs(pos) % 5000
    g = dev(np.random.default_rng(1).normal(size=(1, 1, 3, 64)), torch.float32)
    gx = host(api.rotary(shape, plan, dev(pos), q=g, transpose=True)[0])
    x = host(q)
    for e in range(64):
        x1 = q.clone()
        x1[..., e] += 1.0
        step = host(x1) - x
        y0, y1 = (R.rotate(t, pos[0], freq, layout) for t in (x, host(x1)))
        want = ((y1 - y0) * host(g)).sum(-1)
        np.testing.assert_allclose(gx[..., e] * step[..., e], want, rtol=0, atol=2.0 ** -19)


# ---- attention ----------------------------------------------------------------------------------
class Case:
    """Device tensors of a tree attention, with NaN wherever the call must not look."""

    def __init__(self, dtype, B, hq, hkv, d, cap, lengths, T, counts, seed=0, bias="ratio", parents="tree", scale=1.0):
        rng = np.random.default_rng(seed)
        dt = DT[dtype]
        self.dtype, self.B, self.T = dtype, B, T
        self.shape = api.make_shape(dtype, B, hq, hkv, d, 8, cap, cap)
        self.L, self.n = lengths, counts if counts is not None else [T] * B
        K, V = (rng.normal(size=(B, hkv, cap, d)) for _ in range(2))
        q, k, v = (rng.normal(size=(B, h, T, d)) * s for h, s in ((hq, scale), (hkv, 1.0), (hkv, 1.0)))
        bs = np.where(rng.random((B, hkv, cap)) < 0.2, rng.exponential(1.0, size=(B, hkv, cap)), 0.0)
        if bias == "masked":
            bs[rng.random((B, hkv, cap)) < 0.3] = -np.inf
        if bias == "none_left":
            bs[:] = -np.inf
        if bias == "lowest":
            bs[rng.random((B, hkv, cap)) < 0.5] = LOWEST
        if bias == "all_lowest":
            bs[:] = LOWEST
        bs = bs.astype(np.float32)
        for b in range(B):
            K[b, :, lengths[b]:] = V[b, :, lengths[b]:] = np.nan
            bs[b, :, lengths[b]:] = np.nan
            K[b][bs[b] == -np.inf] = np.nan
            V[b][bs[b] == -np.inf] = np.inf
            q[b, :, self.n[b]:] = k[b, :, self.n[b]:] = v[b, :, self.n[b]:] = np.nan
        self.parents = None
        pr = np.tile(np.arange(-1, T - 1), (B, 1))
        if parents == "tree":
            pr = np.stack([R.random_tree(rng, T) for _ in range(B)])
        elif parents == "forest":
            pr = np.where(rng.random((B, T)) < 0.5, -1, (rng.random((B, T)) * np.arange(T)).astype(int))
            pr[:, 0] = -1
        self.pr = pr
        if parents != "chain":
            self.parents = dev(pr, torch.int32)
        self.q, self.k, self.v = dev(q, dt), dev(k, dt), dev(v, dt)
        bias_t = dev(bs)
        self.use_bias = bias is not None
        self.cache = api.CompressedCache(self.shape, dev(K, dt), dev(V, dt), bias_t, dev(np.array(lengths), torch.int32))
        self.counts = dev(np.array(counts), torch.int32) if counts is not None else None

    def run(self, out=None, workspace=None, stream=None):
        return api.tree_attn(self.cache, self.q, self.k, self.v, self.parents, self.counts, use_bias=self.use_bias, out=out,
                             workspace=workspace, stream=stream)

    def check(self, out, seqs=None, before=None):
        """bf16: each weight and the output rounded by half a step.  Both: logits right to (d + 4) 2^-24 of their sum of
        magnitudes and 2^-22 of the exponent function and the fp32 exponent (below 64 in magnitude: 2^-18); sums over
        all rows to their number of halves steps (in order), at most 2^-24 of the mass each."""
        d, got = self.shape.head_dim, host(out)
        for b in seqs if seqs is not None else range(self.B):
            n, L = self.n[b], self.L[b]
            c = self.cache
            want, mass, size = R.tree_attn(host(self.q[b]), host(c.K_c[b]), host(c.V_c[b]), host(c.bias[b]) if self.use_bias else None,
                                           L, host(self.k[b]), host(self.v[b]), self.pr[b], n)
            logit = (d + 4) * 2.0 ** -24 * size + 2.0 ** -18
            weights = 2 * logit + (L + n) * 2.0 ** -24 + (2.0 ** -8 if self.dtype == "bf16" else 0.0)
            tol = HALF_STEP[self.dtype] * np.abs(want) + weights * (mass + np.abs(want))
            err = np.abs(got[b, :, :n] - want)
            assert (err <= tol).all(), (b, float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
            if before is not None:
                assert torch.equal(out[b, :, n:], before[b, :, n:])


ATTN = [
    # dtype, B, hq, hkv, d, cap, lengths, T, counts
    ("bf16", 1, 1, 1, 64, 1, [1], 1, None),
    ("bf16", 1, 4, 1, 128, 64, [0], 5, None),
    ("bf16", 2, 8, 2, 128, 130, [129, 1], 7, [7, 3]),
    ("bf16", 3, 4, 4, 64, 300, [300, 128, 127], 9, [0, 9, 1]),
    ("bf16", 1, 32, 8, 128, 1000, [999], 32, [31]),
    ("bf16", 2, 16, 2, 128, 700, [640, 513], 16, None),
    ("bf16", 1, 8, 2, 128, 520, [517], 64, [61]),
    ("bf16", 2, 32, 2, 64, 257, [257, 200], 33, [33, 20]),
    ("bf16", 1, 16, 1, 128, 260, [260], 128, [128]),
    ("bf16", 1, 2, 1, 64, 200, [133], 128, [101]),
    ("bf16", 5, 4, 2, 128, 97, [97, 0, 31, 64, 96], 3, [3, 3, 0, 2, 1]),
    ("fp32", 1, 1, 1, 64, 1, [1], 1, None),
    ("fp32", 2, 4, 2, 64, 201, [201, 64], 7, [7, 4]),
    ("fp32", 3, 4, 2, 128, 300, [300, 0, 65], 13, [13, 13, 0]),
    ("fp32", 1, 16, 1, 64, 130, [128], 33, None),
    ("fp32", 1, 8, 8, 128, 700, [653], 128, [127]),
    ("fp32", 2, 32, 2, 128, 70, [70, 63], 2, [1, 2]),
]


@pytest.mark.parametrize("args", ATTN, ids=lambda a: "-".join(str(x).replace(" ", "") for x in a))
@pytest.mark.parametrize("bias,parents", [("ratio", "tree"), (None, "chain"), ("masked", "forest"), ("none_left", "tree"),
                                          ("lowest", "chain"), ("all_lowest", "forest")])
def test_tree_attn(args, bias, parents):
    c = Case(*args, bias=bias, parents=parents)
    before = torch.full_like(c.q, 7.0)
    out = before.clone()
    ws = api.Workspace(S.selkv_tree_attn_workspace_size(c.shape, c.T))
    c.run(out=out, workspace=ws)
    c.check(out, before=before)
    assert ws.errors() == 0
    again = c.run(out=before.clone(), workspace=ws)
    assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_tree_attn_many_short_sequences(dtype):
    rng = np.random.default_rng(5)
    B = 150
    c = Case(dtype, B, 8, 2, 64, 300, [int(x) for x in rng.integers(0, 301, B)], 6, [int(x) for x in rng.integers(0, 7, B)])
    before = torch.full_like(c.q, 3.0)
    c.check(c.run(out=before.clone()), before=before)


@pytest.mark.parametrize("dtype,B,hq,hkv,d,cap,T", [
    ("bf16", 40, 32, 4, 128, 300, 20), ("bf16", 70, 16, 2, 64, 200, 40), ("bf16", 6, 16, 1, 128, 130, 128),
    ("bf16", 300, 8, 8, 128, 90, 3), ("bf16", 1024, 2, 1, 64, 40, 2), ("fp32", 1024, 2, 1, 64, 40, 2),
    ("fp32", 20, 16, 1, 128, 100, 30)])
def test_tree_attn_several_units_a_cta(dtype, B, hq, hkv, d, cap, T):
    """More units than CTAs: a CTA ends some and begins others, and what two share is joined."""
    rng = np.random.default_rng(11)
    c = Case(dtype, B, hq, hkv, d, cap, [int(x) for x in rng.integers(0, cap + 1, B)], T, [int(x) for x in rng.integers(0, T + 1, B)],
             bias="masked")
    before = torch.full_like(c.q, 3.0)
    ws = api.Workspace(S.selkv_tree_attn_workspace_size(c.shape, T))
    out = c.run(out=before.clone(), workspace=ws)
    c.check(out, before=before)
    assert ws.errors() == 0
    assert torch.equal(c.run(out=before.clone(), workspace=ws), out)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_offsets_past_32_bits(dtype):
    """The last head's rows begin past 2^31 elements.  The work is cut by the lengths alone: to the bit what a small cache
    gives."""
    H, d, L, T, far = 8, 128, 777, 6, 2_500_000
    small = Case(dtype, 1, 16, H, d, 1000, [L], T, None)
    want = small.run()
    shape = api.make_shape(dtype, 1, 16, H, d, 8, far, far)
    big = api.CompressedCache(shape, *(torch.empty((1, H, far, d), dtype=DT[dtype], device="cuda") for _ in range(2)),
                              torch.empty((1, H, far), device="cuda"), small.cache.lengths.clone())
    for to, x in ((big.K_c, small.cache.K_c), (big.V_c, small.cache.V_c), (big.bias, small.cache.bias)):
        to[:, :, :L] = x[:, :, :L]
        to[:, :, L:L + 200] = math.nan
    assert torch.equal(api.tree_attn(big, small.q, small.k, small.v, small.parents), want)
    path, accepted = dev(np.array([[0, 2, 3, 5, -1, -1]]), torch.int32), dev(np.array([4]), torch.int32)
    api.tree_commit(big, small.k, small.v, path, accepted)
    at = [0, 2, 3, 5]
    assert int(big.lengths[0]) == L + 4
    assert torch.equal(big.K_c[0, :, L:L + 4], small.k[0][:, at]) and torch.equal(big.V_c[0, :, L:L + 4], small.v[0][:, at])
    assert (big.bias[0, :, L:L + 4] == 0).all() and big.bias[0, :, L + 4:L + 200].isnan().all() and big.K_c[0, :, L + 4:L + 200].isnan().all()


@pytest.mark.parametrize("dtype,T,hq", [("bf16", 4, 8), ("bf16", 24, 8), ("bf16", 64, 8), ("fp32", 3, 4), ("fp32", 24, 4)])
def test_tree_attn_long_cache(dtype, T, hq):
    c = Case(dtype, 1, hq, 2, 128, 20000, [19937], T, None)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [30.0, 300.0])
def test_tree_attn_large_logits(dtype, scale):
    """Running maxima that move by hundreds from tile to tile."""
    c = Case(dtype, 1, 4, 2, 64, 2000, [1990], 9, None, scale=scale)
    q, K = c.q.double(), c.cache.K_c.double()
    s = (q.view(1, 2, 18, 64) @ K[:, :, :1990].transpose(2, 3)).abs().max().item() / 8
    assert s > 4 * scale / 2
    d, got = 64, host(c.run())
    want, mass, size = R.tree_attn(host(c.q[0]), host(c.cache.K_c[0]), host(c.cache.V_c[0]), host(c.cache.bias[0]), 1990,
                                   host(c.k[0]), host(c.v[0]), c.pr[0], 9)
    # exponents of up to `size` in fp32: half a step of them each
    weights = 2 * ((d + 4) * 2.0 ** -24 * size + size * 2.0 ** -22 + 2.0 ** -18) + 2000 * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0)
    tol = HALF_STEP[dtype] * np.abs(want) + np.expm1(weights) * (mass + np.abs(want))
    assert (np.abs(got[0] - want) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_tree_attn_unseen_values_do_not_reach(dtype, what):
    """A value of token 2 that is no number reaches token 2 and those behind it, and in that element alone; an infinite or NaN key
    of a token reaches those that see it."""
    T = 6
    c = Case(dtype, 1, 4, 2, 64, 140, [137], T, None)
    pr = np.array([-1, 0, 0, 1, 2, 4])
    c.pr[0] = pr
    c.parents = dev(pr[None], torch.int32)
    clean = c.run()
    c.v[:, :, 2, 5] = what
    got = c.run()
    hit = [2, 4, 5]
    assert torch.equal(got[:, :, [0, 1, 3]], clean[:, :, [0, 1, 3]])
    keep = [e for e in range(64) if e != 5]
    assert torch.equal(got[:, :, hit][..., keep], clean[:, :, hit][..., keep])
    bad = got[:, :, hit, 5].float()
    assert bool((bad.isnan() if math.isnan(what) else bad == what).all())
    c.v[:, :, 2, 5] = 0.5
    c.k[:, :, 2] = math.nan
    got = c.run()
    assert torch.equal(got[:, :, [0, 1, 3]], clean[:, :, [0, 1, 3]])
    assert bool(got[:, :, hit].float().isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_tree_attn_reports_what_the_host_cannot_see(dtype):
    c = Case(dtype, 2, 4, 2, 64, 70, [70, 33], 5, [5, 5], parents="chain")
    ws = api.Workspace(S.selkv_tree_attn_workspace_size(c.shape, 5))
    want = c.run(workspace=ws)
    assert ws.errors() == 0
    c.cache.lengths.copy_(torch.tensor([99, 33]))
    assert torch.equal(c.run(workspace=ws), want) and ws.errors() == S.SELKV_DEVERR_LENGTH
    c.cache.lengths.copy_(torch.tensor([70, 33]))
    c.counts.copy_(torch.tensor([6, 5]))
    assert torch.equal(c.run(workspace=ws), want) and ws.errors() == S.SELKV_DEVERR_LENGTH
    c.counts.copy_(torch.tensor([-1, 5]))
    got = c.run(out=torch.full_like(want, 2.0), workspace=ws)
    assert torch.equal(got[1], want[1]) and bool((got[0] == 2).all()) and ws.errors() == S.SELKV_DEVERR_LENGTH
    c.counts.copy_(torch.tensor([5, 5]))
    for bad in (3, 4, -2, 1 << 30):
        pr = np.array([[-1, 0, 1, bad, 3]] * 2)
        c.parents = dev(pr, torch.int32)
        got = c.run(workspace=ws)
        assert ws.errors() == S.SELKV_DEVERR_TREE
        c.pr = np.array([[-1, 0, 1, -1, 3]] * 2)
        c.check(got)


def test_tree_attn_one_token_is_a_decode():
    """A tree of one token and a decode that is given its row: the same sums, each within its own tolerance."""
    for dtype in ("bf16", "fp32"):
        c = Case(dtype, 3, 8, 2, 128, 600, [600 - 1, 333, 0], 1, None)
        out = c.run()
        dec = api.decode(c.cache, c.q[:, :, 0].contiguous(), c.k[:, :, 0].contiguous(), c.v[:, :, 0].contiguous())
        err = (out[:, :, 0].double() - dec.double()).abs().max().item()
        assert err <= (2e-2 if dtype == "bf16" else 1e-5) * 2, err


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_tree_attn_streams_graphs_and_shared_workspaces(dtype):
    a = Case(dtype, 2, 8, 2, 128, 900, [900, 411], 8, [8, 5], seed=1)
    b = Case(dtype, 1, 4, 1, 64, 3000, [2999], 40, None, seed=2)
    want = [x.run(out=torch.zeros_like(x.q)) for x in (a, b)]
    size = max(S.selkv_tree_attn_workspace_size(x.shape, x.T) for x in (a, b))
    ws = api.Workspace(size)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream, None):
        outs = [x.run(out=torch.zeros_like(x.q), workspace=ws, stream=stream) for x in (a, b)]
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    # two graphs over one workspace, replayed in turn; inputs change in between
    outs = [torch.zeros_like(x.q) for x in (a, b)]
    graphs = []
    for x, o in zip((a, b), outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run(out=o, workspace=ws)
        graphs.append(g)
    for _ in range(3):
        for g, o, w in zip(graphs, outs, want):
            o.zero_()
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    a.cache.lengths.copy_(torch.tensor([17, 900]))
    a.L = [17, 900]
    a.cache.K_c.nan_to_num_(0.5)
    a.cache.V_c.nan_to_num_(0.5)
    a.cache.bias.nan_to_num_(0.25)
    graphs[0].replay()
    a.check(outs[0])
    # two calls at once, a workspace each
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
    o1 = a.run(out=torch.zeros_like(a.q), stream=side)
    o2 = b.run(out=torch.zeros_like(b.q))
    torch.cuda.synchronize()
    assert torch.equal(o1, outs[0]) and torch.equal(o2, want[1])


def test_helpers_refuse_other_layouts():
    c = Case("bf16", 1, 4, 2, 64, 70, [70], 5, None)
    for kw in (dict(q=c.q.transpose(1, 2)), dict(q=c.q.float()), dict(k=c.k[:, :1]), dict(parents=c.parents.long()),
               dict(parents=c.parents[:, :4]), dict(counts=torch.zeros(2, dtype=torch.int32, device="cuda")), dict(q=c.q.cpu())):
        a = dict(q=c.q, k=c.k, v=c.v, parents=c.parents, counts=None)
        a.update(kw)
        with pytest.raises(S.SelKVError):
            api.tree_attn(c.cache, a["q"], a["k"], a["v"], a["parents"], a["counts"])


# ---- verification -------------------------------------------------------------------------------
def probabilities(rng, shape, sharp):
    x = np.exp(rng.normal(size=shape) * sharp)
    return (x / x.sum(-1, keepdims=True)).astype(np.float32)


def run_verify(tokens, parents, u, target, draft, counts=None, ws=None):
    a, p, x = api.tree_verify(dev(tokens, torch.int32), dev(parents, torch.int32) if parents is not None else None, dev(u), dev(target),
                              dev(draft) if draft is not None else None,
                              dev(np.array(counts), torch.int32) if counts is not None else None, workspace=ws)
    return a.cpu().numpy(), p.cpu().numpy(), x.cpu().numpy()


def check_verify(got, tokens, parents, u, target, draft, counts=None):
    B, T, _ = target.shape
    for b in range(B):
        n = T if counts is None else counts[b]
        pr = parents[b] if parents is not None else np.arange(-1, T - 1)
        a, path, nxt = R.tree_verify(tokens[b], pr, u[b].astype(np.float64), target[b].astype(np.float64),
                                     draft[b].astype(np.float64) if draft is not None else None, n)
        assert got[0][b] == a and list(got[1][b]) == path + [-1] * (T - a) and got[2][b] == nxt, (b, a, path, nxt, got[0][b], got[1][b], got[2][b])


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("B,T,V", [(1, 1, 1), (1, 5, 3), (3, 8, 100), (2, 16, 1023), (2, 6, 4096), (40, 9, 1025), (2, 128, 300), (1, 7, 50001),
                                   (400, 4, 2049)])
def test_tree_verify(drawn, B, T, V):
    rng = np.random.default_rng(V + T + drawn)
    for chain in (False, True):
        target = probabilities(rng, (B, T, V), 2.0)
        draft = probabilities(rng, (B, T, V), 0.0) if V < 4 else None
        noisy = target.astype(np.float64) ** 0.8
        draft = (noisy / noisy.sum(-1, keepdims=True)).astype(np.float32) if draft is None else draft
        parents = None if chain else np.stack([R.random_tree(rng, T, 0.3) for _ in range(B)])
        pr = np.tile(np.arange(-1, T - 1), (B, 1)) if chain else parents
        tokens = np.zeros((B, T), dtype=np.int32)
        for b in range(B):
            for t in range(1, T):
                q = draft[b, pr[b, t]].astype(np.float64)
                tokens[b, t] = rng.choice(V, p=q / q.sum()) if rng.random() < 0.8 else int(target[b, pr[b, t]].argmax())
        u = rng.random((B, T)).astype(np.float32)
        u = np.minimum(u, np.float32(1 - 2.0 ** -24))
        counts = None if chain else [int(x) for x in rng.integers(0, T + 1, B)]
        ws = api.Workspace(S.selkv_tree_verify_workspace_size(B, T, V))
        got = run_verify(tokens, parents, u, target, draft if drawn else None, counts, ws)
        check_verify(got, tokens, parents, u, target, draft if drawn else None, counts)
        assert ws.errors() == 0


@pytest.mark.parametrize("drawn", [True, False])
def test_tree_verify_largest_vocabulary(drawn):
    test_tree_verify(drawn, 1, 4, 1 << 20)


@pytest.mark.parametrize("V", [8, 4096, 40000])
def test_tree_verify_draws_on_the_border(V):
    """Dyadic probabilities: running sums are exact, and a number on the border of two tokens draws the upper one; a
    child whose test is an equality is not accepted."""
    w = np.zeros(V, dtype=np.float32)
    at = np.sort(np.random.default_rng(V).choice(V, 8, replace=False))
    w[at] = np.array([1, 3, 4, 8, 16, 16, 8, 8], dtype=np.float32) / 64
    edges = np.concatenate([[0], np.cumsum(w[at].astype(np.float64))[:-1]])
    us = np.concatenate([edges, edges[1:] - 2.0 ** -24, [1 - 2.0 ** -24, 2.0 ** -30]]).astype(np.float32)
    B = len(us)
    target = np.tile(w, (B, 1, 1))
    got = run_verify(np.zeros((B, 1)), None, us[:, None], target, None)
    want = [at[np.searchsorted(np.cumsum(w[at].astype(np.float64)), float(u), side="right")] for u in us]
    np.testing.assert_array_equal(got[2], want)
    # u q(x) == p(x) exactly: rejected; one step below: accepted
    q = np.zeros(V, dtype=np.float32)
    q[at] = 1 / 8
    x = int(at[1])  # p 3/64, q 1/8: the border is 3/8
    us = np.array([[0.3, 0.375], [0.3, 0.375 - 2.0 ** -24]], dtype=np.float32)
    target, draft = np.tile(w, (2, 2, 1)), np.tile(q, (2, 2, 1))
    tok = np.array([[0, x], [0, x]])
    got = run_verify(tok, None, us, target, draft)
    check_verify(got, tok, None, us, target, draft)
    assert list(got[0]) == [1, 2]


@pytest.mark.parametrize("drawn", [True, False])
def test_tree_verify_rejections_pile_up(drawn):
    """Many children of one node, all but the last rejected; the same token twice; a target without mass beside the
    rejected ones."""
    T, V = 64, 700
    rng = np.random.default_rng(3)
    parents = np.zeros((3, T), dtype=np.int32)
    parents[:, 0] = -1
    target, draft = probabilities(rng, (3, T, V), 0.5), probabilities(rng, (3, T, V), 1.5)
    tokens = rng.integers(0, V, size=(3, T)).astype(np.int32)
    tokens[:, 5] = tokens[:, 4]
    u = np.full((3, T), 1 - 2.0 ** -24, dtype=np.float32)
    u[:, 0] = [0.1, 0.5, 0.9]
    u[1, T - 1] = 0.0
    target[2, 0] = 0
    target[2, 0, tokens[2, 1]] = 1.0  # accepted, or all that is left is what was there
    got = run_verify(tokens, parents, u, target, draft if drawn else None)
    check_verify(got, tokens, parents, u, target, draft if drawn else None)
    # p == q: what is left of a rejection has no mass, and what was there stays
    u[:, 1:] = 0.99
    same = target.copy()
    same[2, 0] = 1.0 / 1024
    got = run_verify(tokens, parents, u, same, same)
    check_verify(got, tokens, parents, u, same, same)


def test_tree_verify_reports_bad_numbers():
    T, V = 4, 500
    rng = np.random.default_rng(4)
    base = dict(target=probabilities(rng, (1, T, V), 1.0), draft=probabilities(rng, (1, T, V), 1.0), tokens=np.array([[0, 3, 5, 7]]),
                parents=np.array([[-1, 0, 0, 0]]), u=np.array([[0.5, 0.999, 0.999, 0.999]], dtype=np.float32))
    ws = api.Workspace(256)

    def got(counts=None, **kw):
        a = {**{k: v.copy() for k, v in base.items()}, **kw}
        out = run_verify(a["tokens"], a["parents"], a["u"], a["target"], a["draft"], counts, ws)
        assert 0 <= out[2][0] < V or out[0][0] == 0
        return out, ws.errors()

    assert got()[1] == 0
    for x in (math.nan, -0.25, math.inf, 2.0):
        t = base["target"].copy()
        t[0, :, 9] = x  # (in every row: the call meets the one of its last node)
        zero = t.copy()
        zero[0, :, 9] = 0.0
        out, flags = got(target=t)
        assert flags == S.SELKV_DEVERR_VALUE
        want, _ = got(target=zero)
        assert all(np.array_equal(p, q) for p, q in zip(out, want))
    for x in (math.nan, 1.0, -0.5, 7.0):
        u = base["u"].copy()
        u[0, 0] = x
        assert got(u=u)[1] == S.SELKV_DEVERR_VALUE
    for x in (-1, V, 1 << 30):
        tok = base["tokens"].copy()
        tok[0, 1] = x
        assert got(tokens=tok)[1] == S.SELKV_DEVERR_VALUE
    assert got(target=np.zeros_like(base["target"]))[0][2][0] == V - 1
    assert ws.errors() == 0
    for x in (1, 2, -5):
        pr = base["parents"].copy()
        pr[0, 1] = x
        assert got(parents=pr)[1] & S.SELKV_DEVERR_TREE
    assert got(counts=[5])[1] == S.SELKV_DEVERR_LENGTH
    out, flags = got(counts=[-1])
    assert flags == S.SELKV_DEVERR_LENGTH and out[0][0] == 0 and out[2][0] == -1 and (out[1] == -1).all()


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("V", [5, 700, 40000])
def test_tree_verify_reports_sums_that_do_not_fit(V, drawn):
    rng = np.random.default_rng(3)
    target, draft = (probabilities(rng, (2, 3, V), 1.0) for _ in range(2))
    target[1] = 1.5  # (sequence 0 stays as it should be)
    tokens, u = np.array([[0, 1, 2]] * 2), np.full((2, 3), 0.875, dtype=np.float32)
    ws = api.Workspace(256)
    out = run_verify(tokens, None, u, target, draft if drawn else None, None, ws)
    assert ws.errors() == S.SELKV_DEVERR_VALUE and 0 <= out[2][1] < V
    check_verify([x[:1] for x in out], tokens[:1], None, u[:1], target[:1], draft[:1] if drawn else None)


# ---- commit -------------------------------------------------------------------------------------
def commit_case(dtype, L, B, hkv, d, cap, T, seed=0, bias=True):
    rng = np.random.default_rng(seed)
    shape = api.make_shape(dtype, B, hkv * 2, hkv, d, 8, cap, cap)
    caches, kn, vn = [], [], []
    for _ in range(L):
        K, V = (dev(rng.normal(size=(B, hkv, cap, d)), DT[dtype]) for _ in range(2))
        bs = dev(rng.random((B, hkv, cap)).astype(np.float32)) if bias else None
        caches.append(api.CompressedCache(shape, K, V, bs, dev(rng.integers(0, cap - T + 1, B), torch.int32)))
        kn.append(dev(rng.normal(size=(B, hkv, T, d)), DT[dtype]))
        vn.append(dev(rng.normal(size=(B, hkv, T, d)), DT[dtype]))
    acc = rng.integers(0, T + 1, B)
    path = np.full((B, T), -1)
    for b in range(B):
        path[b, :acc[b]] = np.sort(rng.choice(T, acc[b], replace=False))
    return caches, kn, vn, path, acc


def clone(c):
    return api.CompressedCache(c.shape, c.K_c.clone(), c.V_c.clone(), c.bias.clone() if c.bias is not None else None, c.lengths.clone())


def expect_commit(caches, kn, vn, path, acc):
    out = []
    for c, k, v in zip(caches, kn, vn):
        w = clone(c)
        for b, n in enumerate(acc):
            n, L = int(n), int(c.lengths[b])
            idx = torch.as_tensor(path[b, :n]).cuda().long()
            w.K_c[b, :, L:L + n], w.V_c[b, :, L:L + n] = k[b][:, idx], v[b][:, idx]
            if w.bias is not None:
                w.bias[b, :, L:L + n] = 0
            w.lengths[b] = L + n
        out.append(w)
    return out


def same_cache(a, b):
    return all(x is None if y is None else torch.equal(x, y) for x, y in ((a.K_c, b.K_c), (a.V_c, b.V_c), (a.bias, b.bias), (a.lengths, b.lengths)))


@pytest.mark.parametrize("dtype,L,B,hkv,d,cap,T,bias", [
    ("bf16", 1, 1, 1, 64, 8, 1, True), ("bf16", 3, 5, 2, 128, 41, 7, True), ("fp32", 2, 3, 3, 64, 200, 33, False),
    ("bf16", 128, 2, 1, 64, 130, 128, True), ("fp32", 33, 1, 2, 128, 64, 5, True), ("bf16", 2, 200, 4, 64, 20, 6, False)])
def test_tree_commit(dtype, L, B, hkv, d, cap, T, bias):
    caches, kn, vn, path, acc = commit_case(dtype, L, B, hkv, d, cap, T, bias=bias)
    want = expect_commit(caches, kn, vn, path, acc)
    ws = api.Workspace(S.selkv_tree_commit_workspace_size(caches[0].shape))
    api.tree_commit(caches, kn, vn, dev(path, torch.int32), dev(acc, torch.int32), workspace=ws)
    assert all(same_cache(c, w) for c, w in zip(caches, want))
    assert ws.errors() == 0


def test_tree_commit_that_does_not_fit():
    caches, kn, vn, path, acc = commit_case("bf16", 2, 4, 2, 64, 50, 6)
    acc[:] = 4
    path[:] = [0, 1, 3, 5, -1, -1]
    caches[0].lengths.copy_(torch.tensor([46, 47, 50, 3]))
    caches[1].lengths.copy_(torch.tensor([1, 2, 46, 49]))
    ws = api.Workspace(256)
    fits = [np.array([4, 0, 0, 4]), np.array([4, 4, 4, 0])]
    want = [expect_commit([c], [k], [v], path, f)[0] for c, k, v, f in zip(caches, kn, vn, fits)]
    p = dev(path, torch.int32)
    api.tree_commit(caches, kn, vn, p, dev(acc, torch.int32), workspace=ws)
    assert all(same_cache(c, w) for c, w in zip(caches, want))
    assert ws.errors() == S.SELKV_DEVERR_CAPACITY
    # a path that names no token: none of the sequence's rows
    for c in caches:
        c.lengths.fill_(10)
    p[1, 2] = 6
    p[2, 0] = -1
    want = expect_commit(caches, kn, vn, path, np.array([4, 0, 0, 4]))
    api.tree_commit(caches, kn, vn, p, dev(acc, torch.int32), workspace=ws)
    assert all(same_cache(c, w) for c, w in zip(caches, want))
    assert ws.errors() == S.SELKV_DEVERR_TREE
    # counts and lengths out of range
    p = dev(np.tile(np.arange(6), (4, 1)), torch.int32)
    for c in caches:
        c.lengths.copy_(torch.tensor([10, 20, -3, 51]))
    before = [clone(c) for c in caches]
    for c in before:
        c.lengths.copy_(torch.tensor([10, 20, 0, 50]))
    want = expect_commit(before, kn, vn, np.tile(np.arange(6), (4, 1)), np.array([6, 0, 2, 0]))
    for c in want:
        c.lengths[3] = 51
    api.tree_commit(caches, kn, vn, p, dev(np.array([9, -1, 2, 0]), torch.int32), workspace=ws)
    assert all(same_cache(c, w) for c, w in zip(caches, want))
    assert ws.errors() == S.SELKV_DEVERR_LENGTH


# ---- a run of them together ---------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("graph", [False, True])
def test_speculative_steps(dtype, graph):
    """Steps of drafting, rotation, tree attention, verification and commit, then a decode over what they left: the
    accepted tokens one by one through plain decodes give the same outputs and the same cache."""
    rng = np.random.default_rng(9)
    B, hq, hkv, d, T, V, steps, layers = 2, 8, 2, 64, 7, 50, 4, 2
    cap, n0 = 400, [300, 211]
    shape = api.make_shape(dtype, B, hq, hkv, d, 8, cap, cap)
    caches = []
    for _ in range(layers):
        K, V_ = (dev(rng.normal(size=(B, hkv, cap, d)), DT[dtype]) for _ in range(2))
        caches.append(api.CompressedCache(shape, K, V_, dev(rng.random((B, hkv, cap)).astype(np.float32)), dev(np.array(n0), torch.int32)))
    plain = [clone(c) for c in caches]
    plan = api.rotary_plan(d, layout="half")
    size = max(S.selkv_tree_attn_workspace_size(shape, T), S.selkv_tree_verify_workspace_size(B, T, V))
    ws, dws = api.Workspace(size), api.Workspace(S.selkv_decode_workspace_size(shape))
    # inputs of a step, filled in place
    parents = torch.empty((B, T), dtype=torch.int32, device="cuda")
    tokens, positions = torch.empty_like(parents), torch.empty_like(parents)
    u = torch.empty((B, T), device="cuda")
    target, draft = torch.empty((B, T, V), device="cuda"), torch.empty((B, T, V), device="cuda")
    q = [torch.empty((B, hq, T, d), dtype=DT[dtype], device="cuda") for _ in range(layers)]
    k, v = ([torch.empty((B, hkv, T, d), dtype=DT[dtype], device="cuda") for _ in range(layers)] for _ in range(2))
    outs = [torch.zeros_like(x) for x in q]
    res = tuple(torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((B,), (B, T), (B,)))

    def step():
        for i in range(layers):
            api.rotary(shape, plan, positions, q[i], k[i], out=(q[i], k[i]))
            api.tree_attn(caches[i], q[i], k[i], v[i], parents, out=outs[i], workspace=ws)
        api.tree_verify(tokens, parents, u, target, draft, out=res, workspace=ws)
        api.tree_commit(caches, k, v, res[1], res[0], workspace=ws)

    g = None
    total = 0
    for s in range(steps):
        pr = np.stack([R.random_tree(rng, T, 0.6) for _ in range(B)])
        depth = np.zeros((B, T), dtype=np.int64)
        for t in range(1, T):
            depth[:, t] = depth[np.arange(B), pr[:, t]] + 1
        pos = caches[0].lengths.cpu().numpy()[:, None] + depth
        tp = probabilities(rng, (B, T, V), 1.0)
        dp = probabilities(rng, (B, T, V), 0.1)
        tok = np.zeros((B, T))
        for b in range(B):
            for t in range(1, T):
                tok[b, t] = rng.choice(V, p=(lambda z: z / z.sum())(tp[b, pr[b, t]].astype(np.float64)))
        raw = [[rng.normal(size=(B, h, T, d)) for h in (hq, hkv, hkv)] for _ in range(layers)]

        def fill():
            for dst, src in ((parents, pr), (tokens, tok), (positions, pos), (u, rng.random((B, T)) * 0.999), (target, tp), (draft, dp)):
                dst.copy_(torch.as_tensor(src))
            for i in range(layers):
                for dst, src in zip((q[i], k[i], v[i]), raw[i]):
                    dst.copy_(torch.as_tensor(src))
        fill()
        if graph and g is None:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
        if graph:
            g.replay()
        else:
            step()
        acc, path = res[0].cpu().numpy(), res[1].cpu().numpy()
        total += int((acc - 1).sum())
        check_verify([r.cpu().numpy() for r in res], tok.astype(int), pr, u.cpu().numpy(), tp, dp)
        # the same rows one at a time, sequence by sequence
        for i in range(layers):
            for j in range(int(acc.max())):
                at = np.where(j < acc, path[:, min(j, T - 1)], 0)
                idx = torch.as_tensor(at).cuda()
                pick = lambda x: x[torch.arange(B, device="cuda"), :, idx].contiguous()  # noqa: E731
                keep = clone(plain[i])
                out = api.decode(plain[i], pick(q[i]), pick(k[i]), pick(v[i]), workspace=dws)
                for b in range(B):
                    if j < acc[b]:
                        err = (out[b].double() - outs[i][b, :, at[b]].double()).abs().max().item()
                        assert err <= (4e-2 if dtype == "bf16" else 2e-5), (s, i, j, b, err)
                    else:  # this sequence's path ended before: its row is taken back
                        for x, y in ((plain[i].K_c, keep.K_c), (plain[i].V_c, keep.V_c), (plain[i].bias, keep.bias), (plain[i].lengths, keep.lengths)):
                            x[b] = y[b]
            assert same_cache(plain[i], caches[i]), (s, i)
        assert ws.errors() == 0 and dws.errors() == 0
    assert total > 0


@pytest.mark.parametrize("trial", range(20))
def test_decode_directly_after_a_commit(trial):
    """A decode comes up while the kernel before it still runs: right behind a commit it has to see the new rows."""
    caches, kn, vn, path, acc = commit_case("bf16", 4, 4, 4, 128, 2100, 64, seed=trial)
    want = expect_commit(caches, kn, vn, path, acc)
    q = dev(np.random.default_rng(trial).normal(size=(4, 8, 128)), torch.bfloat16)
    ws, dws = api.Workspace(256), api.Workspace(S.selkv_decode_workspace_size(caches[0].shape))
    p, n = dev(path, torch.int32), dev(acc, torch.int32)
    ref = [api.decode(c, q, workspace=dws) for c in want]
    torch.cuda.synchronize()
    api.tree_commit(caches, kn, vn, p, n, workspace=ws)
    got = [api.decode(c, q, workspace=dws) for c in caches]
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
