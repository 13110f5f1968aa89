"""Caches held in 8 bits at their edges, against the plain form in 64 bits: workspaces that go from one cache to
another, weights far below the largest, a NaN among the compensation, scales of the caller's own
below the smallest fresh one, rows read back and decoded over at once, and fp32 decodes held to a limit that tells queries and
weights in two halves from one."""
import math

import numpy as np
import pytest
import torch

import paper_2607_16213_gb300 as S
from paper_2607_16213_gb300 import api
import quant_fine as F
import quant_ref as R
from test_gpu_quant import Model, TORCH, filled, gen, make, np64, rows, u8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_16213_gb300 import build as b
    b.build()
    S.library()


# ---- one workspace, many caches -------------------------------------------------------------------------
@pytest.mark.parametrize("shapes", [
    [(4, 16384, 16000), (4, 4096, 3000)],
    [(8, 32768, 5000), (8, 4096, 4000)],
    [(1, 32768, 30000), (64, 1024, 700), (3, 9000, 8000)],
])
def test_a_workspace_goes_from_cache_to_cache(shapes):
    """Tokens decoded in turn over caches of other capacities and batches on one workspace: outputs, lengths and
    codes are those of calls with a workspace of their own."""
    hq, hkv, d = 32, 8, 128
    def caches():
        return [filled("bf16", B, hq, hkv, d, cap, "e4m3", 64, [n - 11 * b for b in range(B)], cap)[0] for B, cap, n in shapes]
    shared, alone = caches(), caches()
    size = max(S.selkv_decode_q_workspace_size(c.shape) for c in shared)
    ws = api.Workspace(size)
    g = gen(41)
    for turn in range(3):
        for one, two in zip(shared, alone):
            B = one.shape.batch
            q = torch.randn((B, hq, d), generator=g, device="cuda").bfloat16()
            k, v = (torch.randn((B, hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
            got = api.decode_quant(one, q, k, v, out=torch.full_like(q, math.nan), workspace=ws)
            want = api.decode_quant(two, q, k, v)
            assert torch.equal(got, want), (turn, B)
            assert torch.equal(one.lengths, two.lengths)
            for x, y in ((one.K, two.K), (one.V, two.V), (one.K_scale, two.K_scale), (one.V_scale, two.V_scale)):
                assert torch.equal(x.view(torch.int8), y.view(torch.int8))
    assert ws.errors() == 0


def test_a_decode_workspace_serves_append_and_read():
    """The three calls on one workspace, the decodes' partials between them."""
    B, hq, hkv, d = 3, 16, 4, 128
    c, g = filled("bf16", B, hq, hkv, d, 9000, "int8", 64, [8000, 7000, 20], 6)
    model = Model(c)
    ws = api.Workspace(S.selkv_decode_q_workspace_size(c.shape))
    for turn in range(3):
        q = torch.randn((B, hq, d), generator=g, device="cuda").bfloat16()
        k, v = rows(g, B, hkv, 5, d, "bf16"), rows(g, B, hkv, 5, d, "bf16")
        api.quant_append(c, k, v, workspace=ws)
        model.append(k, v, [5] * B)
        kn, vn = (torch.randn((B, hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
        api.decode_quant(c, q, kn, vn, workspace=ws)
        model.append(kn[:, :, None], vn[:, :, None], [1] * B)
        K, _ = api.quant_read(c, 16, 100, workspace=ws)
        assert torch.equal(K[0, 1].cpu(), torch.from_numpy(model.head(0, 1)[0][16:116]).bfloat16())
    model.check()
    assert ws.errors() == 0


# ---- weights far below the largest --------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("gap", [90, 109, 112, 115, 118, 121, 124])
@pytest.mark.parametrize("B,hkv,n", [(40, 8, 700), (5, 2, 5000)])
def test_decode_weights_far_below_the_largest(kind, dtype, zeros, gap, B, hkv, n):
    """Sixteen rows of values around 1 (or 0) with the largest logit, sixteen of values around 2^122 (or 2^10) with one `gap`
    (in base 2) below: their share, weights above 2^-126 of the largest times huge values, is (all of) the output.
    In the other half of a tile, in another tile of a warp, of a CTA or (few, long caches) of the batch, before and behind.

    What it may be off, with u = 2^-24: the bias in base 2 is rounded twice (the constant, the product) and the difference of
    two logits once, numbers below 128, so 3 x 64 u ln 2 = 133 u of a weight, and the exponential 4 u; both again for the
    normaliser.  The units of the output and their fold: up to seven roundings of exponents below 256, 128 u ln 2 each, and
    three exponentials: 633 u.  The weight in fp16 (2^-11; fp32 2^-21), sums of 32 products of positive numbers cut off, 64 u, folds
    200 u, and the output's own rounding.  Codes of rows that count are three quarters of the largest and more."""
    hq, d, block = hkv, 64, 16
    at = {0: (0, 16), 1: (16, 0), 2: (0, 256), 3: (256, 0), 4: (640, 32)}  # first row of the large logits, of the others
    c = make(dtype, B, hq, hkv, d, n + 20, kind, block)
    g = gen(gap)
    small, huge = (0.0, 2.0 ** 10) if zeros else (1.0, 2.0 ** 122)
    V = torch.zeros((B, hkv, n, d), device="cuda")
    bias = torch.full((B, hkv, n), -math.inf, device="cuda")
    for b in range(B):
        top, far = at[b % len(at)]
        V[b, :, top:top + 16] = small * (0.75 + torch.rand((hkv, 16, d), generator=g, device="cuda") / 4)
        V[b, :, far:far + 16] = huge * (0.75 + torch.rand((hkv, 16, d), generator=g, device="cuda") / 4)
        bias[b, :, top:top + 16] = 0.0
        bias[b, :, far:far + 16] = -gap * math.log(2)
    K = torch.zeros_like(V)
    api.quant_append(c, K.to(TORCH[dtype]), V.to(TORCH[dtype]), bias)
    model = Model(c)
    q = torch.randn((B, hq, d), generator=g, device="cuda").to(TORCH[dtype])
    ws = api.Workspace(S.selkv_decode_q_workspace_size(c.shape))
    got = np64(api.decode_quant(c, q, workspace=ws))
    assert ws.errors() == 0
    u = 2.0 ** -24
    lim = (2 * 137 + 633 + 264) * u + (2.0 ** -11 + 2.0 ** -8 if dtype == "bf16" else 2.0 ** -21 + u)
    for b in range(B):
        for h in range(hkv):
            kk, vv = model.head(b, h)
            live = np.isfinite(model.bias[b, h, :n])
            want = R.decode_head(np64(q)[b, h:h + 1], kk[live], vv[live], model.bias[b, h, :n][live])[0][0]
            err = np.abs(got[b, h] - want) / want
            assert err.max() <= lim, (b, h, float(err.max()), lim, got[b, h, :3], want[:3])


# ---- compensation that is no number ---------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,hq", [("bf16", 4), ("bf16", 24), ("fp32", 4), ("fp32", 20)])
@pytest.mark.parametrize("cap", [300, 9000])
def test_decode_nan_bias(kind, dtype, hq, cap):
    """A NaN in the bias of a row makes the outputs of its KV head's query heads NaN, as the formula does, and no other; also beside
    rows without weight, and where it is the only row that is not masked."""
    B, hkv, d = 4, 2, 64
    lens = [cap - 20, cap - 60, 31, 1]
    c, g = filled(dtype, B, hq, hkv, d, cap, kind, 32, lens, cap)
    c.bias[0, 1, 100] = math.nan
    c.bias[1, 0, :] = -math.inf
    c.bias[1, 0, 200] = math.nan
    c.bias[2, 1, :31] = torch.finfo(torch.float32).min
    c.bias[2, 1, 30] = math.nan
    c.bias[3, 0, 0] = math.nan
    c.bias[3, 1, 1:] = math.nan  # behind the rows of the cache: not read
    q = torch.randn((B, hq, d), generator=g, device="cuda").to(TORCH[dtype])
    out = api.decode_quant(c, q).view(B, hkv, hq // hkv, d)
    want = torch.zeros((B, hkv), dtype=torch.bool, device="cuda")
    want[0, 1] = want[1, 0] = want[2, 1] = want[3, 0] = True
    assert torch.equal(out.isnan().all(-1).all(-1), want) and torch.equal(out.isnan().any(-1).any(-1), want)


# ---- scales of the caller's own -------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("by", ["append", "decode"])
@pytest.mark.parametrize("e0", [-126, -110, -101, -100, 20])
def test_rows_behind_a_callers_scale(kind, dtype, by, e0):
    """A block with rows and a scale that the caller set, any normal number: the scale is kept or grows by the smallest power of
    two that covers the new row, and the old codes are rounded to it."""
    B, H, d, block, L = 5, 2, 64, 32, 10
    c = make(dtype, B, H, H, d, 64, kind, block, junk=False)
    s0 = 2.0 ** e0
    g = gen(e0 + 200)
    code = torch.randint(-100, 101, (B, H, L, d), generator=g, device="cuda")
    for t, s in ((c.K, c.K_scale), (c.V, c.V_scale)):
        t[:, :, :L] = code.to(torch.int8) if kind == "int8" else code.float().to(torch.float8_e4m3fn)
        s[:, :, 0] = s0
    c.lengths.fill_(L)
    # largest magnitudes of the new rows, in units of the scale: within its codes, and 1, 2, 5 and 30 doublings past them
    most = R.QMAX[kind] * torch.tensor([0.5, 1.5, 3.0, 30.0, 2.0 ** 29 * 1.1], device="cuda")
    x = (torch.rand((B, H, d), generator=g, device="cuda") - 0.5) * most[:, None, None]
    x[:, :, 7] = most[:, None]
    x = (x.double() * s0).to(TORCH[dtype])
    old = [R.values(u8(t), kind)[:, :, :L] for t in (c.K, c.V)]
    if by == "append":
        api.quant_append(c, x[:, :, None].contiguous(), (-x)[:, :, None].contiguous())
    else:
        api.decode_quant(c, torch.zeros((B, H, d), dtype=TORCH[dtype], device="cuda"), x, -x)
    assert c.lengths.tolist() == [L + 1] * B
    for t, s, was, new in ((c.K, c.K_scale, old[0], np64(x)), (c.V, c.V_scale, old[1], -np64(x))):
        got, scale = R.values(u8(t), kind), np64(s)
        for b in range(B):
            for h in range(H):
                want = s0
                while want * R.QMAX[kind] < np.abs(new[b, h]).max():
                    want *= 2
                assert scale[b, h, 0] == want
                np.testing.assert_array_equal(got[b, h, :L], R.round_code(was[b, h] * (s0 / want), kind))
                np.testing.assert_array_equal(got[b, h, L], R.round_code(new[b, h] / want, kind))


# ---- rows read back, then decoded over ------------------------------------------------------------------
@pytest.mark.parametrize("graph", [False, True])
def test_the_kernel_in_front_of_a_decode_writes_no_rows(graph):
    """A bf16 decode loads rows before it waits for the kernel in front of it: a read's rows are written by an earlier one of its two.
    Reads of several caches into the same rows, a decode behind each, on a stream of their own and captured."""
    B, hq, hkv, d, cap = 2, 16, 4, 128, 6000
    shape = api.make_shape("bf16", B, hq, hkv, d, 32, cap, cap)
    g = gen(61)
    q = torch.randn((B, hq, d), generator=g, device="cuda").bfloat16()
    caches = [filled("bf16", B, hq, hkv, d, cap, "int8", 64, [cap - 3 * i, cap - 500], i)[0] for i in range(3)]
    full = api.alloc_compressed(shape)
    full.lengths.fill_(cap - 501)
    ws, wr = api.Workspace(S.selkv_decode_workspace_size(shape)), api.Workspace(S.selkv_qcache_workspace_size(shape))
    outs = torch.empty((12, B, hq, d), dtype=torch.bfloat16, device="cuda")

    def one(i, out, wait=False):
        before = S.selkv_kernel_launches()
        api.quant_read(caches[i % 3], out=(full.K_c, full.V_c), workspace=wr)
        assert S.selkv_kernel_launches() == before + 2
        if wait:
            torch.cuda.synchronize()
        api.decode(full, q, use_bias=False, out=out, workspace=ws, stream=torch.cuda.current_stream().cuda_stream)

    want = torch.empty_like(outs[:3])
    for i in range(3):
        one(i, want[i], wait=True)
    torch.cuda.synchronize()
    assert not torch.equal(want[0], want[1])
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        if graph:
            recorded = torch.cuda.CUDAGraph()
            with torch.cuda.graph(recorded, stream=stream):
                for i in range(12):
                    one(i, outs[i])
            for _ in range(3):
                outs.fill_(math.nan)
                recorded.replay()
        else:
            for i in range(12):
                one(i, outs[i])
    torch.cuda.synchronize()
    for i in range(12):
        assert torch.equal(outs[i], want[i % 3]), i
    assert ws.errors() == 0 and wr.errors() == 0


# ---- fp32 caches: both halves count ---------------------------------------------------------------------
@pytest.mark.parametrize("case", F.CASES)
@pytest.mark.parametrize("seed", [1, 2])
def test_fp32_decode_to_its_last_digits(case, seed):
    """Unit rows and queries (F says what a result may be off; the host test beside it that one half would not do)."""
    d, hq, hkv, lens, kind, block = case
    q, k, v, bias = (torch.from_numpy(x).cuda() for x in F.inputs(case, seed))
    B, n = len(lens), max(lens)
    c = make("fp32", B, hq, hkv, d, n + 5, kind, block)
    api.quant_append(c, k, v, bias, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    model = Model(c)
    out = np64(api.decode_quant(c, q)).reshape(B, hkv, hq // hkv, d)
    worst = 0.0
    for b in range(B):
        for h in range(hkv):
            kk, vv = model.head(b, h)
            np.testing.assert_array_equal(kk, F.cached(np64(k)[b, h], lens[b], kind, block)[0])
            want, lim = F.limit(np64(q)[b].reshape(hkv, -1, d)[h], kk, vv, model.bias[b, h, :lens[b]])
            worst = max(worst, float((np.abs(out[b, h] - want) / lim).max()))
    print("largest error over its limit: %.3f" % worst)
    assert worst <= 1


# ---- the most sequences, and streams by their handles ---------------------------------------------------
@pytest.mark.parametrize("kind,d", [("e4m3", 64), ("int8", 128)])
def test_the_most_sequences_and_heads(kind, d):
    """1024 sequences of 32 KV heads on one workspace: appended to, decoded over with a new row, read back."""
    B, hkv, cap = 1024, 32, 50
    c = make("bf16", B, hkv, hkv, d, cap, kind, 16)
    g = gen(d)
    k, v = rows(g, B, hkv, 40, d, "bf16", loud=False), rows(g, B, hkv, 40, d, "bf16", loud=False)
    counts = (torch.arange(B, dtype=torch.int32, device="cuda") * 7) % 41
    ws = api.Workspace(S.selkv_decode_q_workspace_size(c.shape))
    api.quant_append(c, k, v, counts=counts, workspace=ws)
    assert torch.equal(c.lengths, counts)
    K, V = (x.double() for x in api.quant_read(c, 0, 41, workspace=ws))
    q = torch.randn((B, hkv, d), generator=g, device="cuda").bfloat16()
    kn, vn = (torch.randn((B, hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    out = api.decode_quant(c, q, kn, vn, workspace=ws)
    assert torch.equal(c.lengths, counts + 1) and ws.errors() == 0
    at = counts.long()[:, None, None, None].expand(B, hkv, 1, d)
    K.scatter_(2, at, kn.double()[:, :, None])
    V.scatter_(2, at, vn.double()[:, :, None])
    s = (q.double()[:, :, None] * K).sum(3) / math.sqrt(d)
    s.masked_fill_(torch.arange(41, device="cuda") > counts[:, None, None], -math.inf)
    p = torch.softmax(s, 2)
    want = (p[..., None] * V).sum(2)
    # The rows read back in bf16 are off by 2^-8 of themselves (int8 codes times four bits; e4m3 exactly): of a key that moves
    # a logit by 2^-8 sum |q k| / sqrt(d), and a weight and the normaliser by e to that.  The kernel: weights 2^-11, logits and sums
    # far below 2^-11; the output 2^-8.
    read = 2.0 ** -8 if kind == "int8" else 0.0
    mag = (q.double().abs()[:, :, None] * K.abs()).sum(3).amax(2) / math.sqrt(d)
    pv = (p[..., None] * V.abs()).sum(2)
    lim = ((read + torch.expm1(2 * read * mag))[..., None] + 2.0 ** -11 + 2.0 ** -11 * (1 + mag)[..., None]) * pv + 2.0 ** -8 * want.abs() + 1e-30
    assert bool(((out.double() - want).abs() <= lim).all())


def test_streams_by_handle_and_object():
    """Every call takes a stream as its handle (0: the default one) or as an object."""
    c, g = filled("bf16", 2, 8, 2, 128, 300, "e4m3", 64, [250, 30], 12)
    model = Model(c)
    q = torch.randn((2, 8, 128), generator=g, device="cuda").bfloat16()
    want = api.decode_quant(c, q)
    torch.cuda.synchronize()
    for stream in (0, torch.cuda.default_stream(), torch.cuda.Stream(), torch.cuda.Stream().cuda_stream):
        k, v = rows(g, 2, 2, 3, 128, "bf16"), rows(g, 2, 2, 3, 128, "bf16")
        torch.cuda.synchronize()
        out = api.decode_quant(c, q, stream=stream)
        K, _ = api.quant_read(c, 0, 30, stream=stream)
        api.quant_append(c, k, v, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        for b in range(2):
            assert torch.equal(K[b, 1].cpu(), torch.from_numpy(model.head(b, 1)[0][:30]).bfloat16())
        model.append(k, v, [3, 3])
        model.check()
        want = api.decode_quant(c, q)
        torch.cuda.synchronize()
