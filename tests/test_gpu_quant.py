"""Caches held in 8 bits on the GPU against the plain form in 64 bits (quant_ref.py): written rows
exactly (codes, scales, bias, lengths, and all that a call leaves alone), rows read back exactly, decode within
bounds that count its roundings."""
import math

import numpy as np
import pytest
import torch

import paper_2607_16213_gb300 as S
from paper_2607_16213_gb300 import api
import quant_ref as R

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_16213_gb300 import build as b
    b.build()
    S.library()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rows(g, B, H, n, d, dtype, loud=True):
    """Rows of unequal magnitude, some large, some tiny, some of zeros."""
    x = torch.randn((B, H, n, d), generator=g, device="cuda")
    if loud and n:
        x *= torch.exp(1.5 * torch.randn((B, H, n, 1), generator=g, device="cuda"))
        x *= (torch.rand((B, H, n, 1), generator=g, device="cuda") > 0.03)
    return x.to(TORCH[dtype])


def np64(t):
    return t.double().cpu().numpy()


def u8(codes):
    return codes.view(torch.uint8).cpu().numpy()


def make(dtype, B, hq, hkv, d, cap, kind, block, bias=True, junk=True):
    """An empty cache whose tensors hold junk: codes 0x7f (an e4m3 NaN), NaN scales and bias."""
    shape = api.make_shape(dtype, B, hq, hkv, d, 32, cap, cap)
    c = api.alloc_quant(shape, kind, block, bias)
    if junk:
        for t in (c.K, c.V):
            t.view(torch.uint8).fill_(0x7f)
        for t in (c.K_scale, c.V_scale) + ((c.bias,) if bias else ()):
            t.fill_(math.nan)
    return c


class Model:
    """The same cache in plain form."""

    def __init__(self, c):
        self.c, self.kind, self.block = c, c.cache_type, c.block
        self.K, self.V = R.values(u8(c.K), self.kind), R.values(u8(c.V), self.kind)
        self.ks, self.vs = np64(c.K_scale), np64(c.V_scale)
        self.bias = np64(c.bias) if c.bias is not None else None
        self.L = c.lengths.cpu().numpy().copy()

    def append(self, k, v, counts, bias=None):
        k, v = np64(k), np64(v)
        for b, n in enumerate(counts):
            L = self.L[b]
            if L + n > self.K.shape[2]:
                continue
            for h in range(self.K.shape[1]):
                R.append_head(self.K[b, h], self.ks[b, h], k[b, h, :n], L, self.block, self.kind)
                R.append_head(self.V[b, h], self.vs[b, h], v[b, h, :n], L, self.block, self.kind)
            if self.bias is not None:
                self.bias[b, :, L:L + n] = 0.0 if bias is None else np64(bias)[b, :, :n]
            self.L[b] += n

    def head(self, b, h):
        at = np.arange(self.L[b]) // self.block
        return self.K[b, h, :self.L[b]] * self.ks[b, h][at, None], self.V[b, h, :self.L[b]] * self.vs[b, h][at, None]

    def check(self):
        c = self.c
        np.testing.assert_array_equal(R.values(u8(c.K), self.kind), self.K)
        np.testing.assert_array_equal(R.values(u8(c.V), self.kind), self.V)
        np.testing.assert_array_equal(np64(c.K_scale), self.ks)
        np.testing.assert_array_equal(np64(c.V_scale), self.vs)
        if self.bias is not None:
            np.testing.assert_array_equal(np64(c.bias), self.bias)
        np.testing.assert_array_equal(c.lengths.cpu().numpy(), self.L)


# ---- writing --------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,d,block,B,H,cap,chunks", [
    ("bf16", 128, 64, 1, 2, 400, [[300], [1], [1], [63], [17]]),
    ("bf16", 128, 16, 3, 2, 133, [[0, 7, 100], [16, 1, 0], [5, 0, 33]]),
    ("bf16", 64, 128, 2, 3, 515, [[129, 1], [1, 126], [255, 1], [3, 300]]),
    ("bf16", 64, 32, 5, 1, 64, [[0, 1, 31, 32, 63], [64, 63, 33, 32, 1]]),
    ("fp32", 128, 32, 2, 2, 257, [[257, 130], [0, 127]]),
    ("fp32", 64, 16, 2, 1, 300, [[17, 200], [1, 1], [1, 1], [120, 90]]),
    ("bf16", 128, 128, 1, 32, 1000, [[999], [1]]),
    ("bf16", 128, 64, 70, 1, 40, [[i % 40 for i in range(70)], [1] * 70]),
])
def test_append(kind, dtype, d, block, B, H, cap, chunks):
    g = gen(d + block + cap)
    c = make(dtype, B, 2 * H, H, d, cap, kind, block)
    model = Model(c)
    ws = api.Workspace(S.selkv_qcache_workspace_size(c.shape))
    for i, counts in enumerate(chunks):
        T = max(max(counts), 1) + i % 3
        k, v = rows(g, B, H, T, d, dtype), rows(g, B, H, T, d, dtype)
        bias = torch.rand((B, H, T), generator=g, device="cuda") if i % 2 == 0 else None
        api.quant_append(c, k, v, bias, torch.tensor(counts, dtype=torch.int32, device="cuda"), workspace=ws)
        assert ws.errors() == 0
        model.append(k, v, counts, bias)
        model.check()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_append_all_rows_without_counts_or_bias(kind):
    g = gen(5)
    c = make("bf16", 2, 4, 2, 64, 200, kind, 64, bias=False)
    model = Model(c)
    for T in (1, 64, 100):
        k, v = rows(g, 2, 2, T, 64, "bf16"), rows(g, 2, 2, T, 64, "bf16")
        api.quant_append(c, k, v)
        model.append(k, v, [T, T])
        model.check()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_special_values(kind, dtype):
    """Infinities, NaN, zeros, the largest and smallest magnitudes, and borders between two codes."""
    c = make(dtype, 1, 1, 1, 64, 256, kind, 16)
    model = Model(c)
    top = torch.finfo(TORCH[dtype]).max
    x = torch.zeros((1, 1, 112, 64), device="cuda")
    g = gen(1)
    x[0, 0, 0:16] = torch.randn((16, 64), generator=g, device="cuda")
    x[0, 0, 3, 5], x[0, 0, 4, 6], x[0, 0, 5, 7] = math.inf, -math.inf, math.nan
    x[0, 0, 16, 0] = math.nan                                           # a block of zeros and a NaN
    x[0, 0, 32:48] = torch.randn((16, 64), generator=g, device="cuda") * top / 8
    x[0, 0, 33, 1], x[0, 0, 34, 2] = top, -top
    x[0, 0, 48:64] = torch.randn((16, 64), generator=g, device="cuda") * 1e-38   # tiny, some subnormal
    x[0, 0, 64:80] = (torch.arange(1024, device="cuda").view(16, 64) - 512) / 4.0  # quarters: borders
    x[0, 0, 80:96] = 2.0 ** -99 * torch.rand((16, 64), generator=g, device="cuda")  # around the smallest scale
    x[0, 0, 96:112] = 1.75 * 2.0 ** -(torch.arange(1024, device="cuda").view(16, 64) % 40)
    x = x.to(TORCH[dtype])
    ws = api.Workspace(S.selkv_qcache_workspace_size(c.shape))
    with np.errstate(invalid="ignore"):
        model.append(x, -x, [112])
        api.quant_append(c, x, -x, workspace=ws)
        assert ws.errors() == S.SELKV_DEVERR_VALUE
        model.check()
        # one more row, larger by far than what its block holds, and one into a block of zeros
        for big in (0.0, top):
            y = torch.full((1, 1, 1, 64), big, device="cuda").to(TORCH[dtype])
            model.append(y, y, [1])
            api.quant_append(c, y, y, workspace=ws)
            assert ws.errors() == 0
            model.check()


@pytest.mark.parametrize("kind,dtype,B,H,d,block", [("int8", "bf16", 40, 32, 64, 32), ("e4m3", "fp32", 70, 8, 128, 128),
                                                  ("e4m3", "bf16", 90, 16, 128, 16)])
def test_append_of_many_tiles(kind, dtype, B, H, d, block):
    """So many tiles that a CTA takes several of them: ragged prompts, then a chunk behind them; a NaN in one."""
    g = gen(B)
    cap, n0, n1 = 700, 500, 190
    c = make(dtype, B, H, H, d, cap, kind, block)
    model = Model(c)
    ws = api.Workspace(S.selkv_qcache_workspace_size(c.shape))
    for n in (n0, n1):
        k, v = rows(g, B, H, n, d, dtype), rows(g, B, H, n, d, dtype)
        counts = [(i * 97) % (n + 1) for i in range(B)]
        counts[B // 2] = n
        v[B // 2, H - 1, n - 1, 5] = math.nan
        api.quant_append(c, k, v, None, torch.tensor(counts, dtype=torch.int32, device="cuda"), workspace=ws)
        assert ws.errors() == S.SELKV_DEVERR_VALUE
        model.append(k, v, counts)
        model.check()


def test_append_flags():
    """Rows that do not fit are not written, lengths and counts out of range are clamped; both are said."""
    g = gen(2)
    c = make("bf16", 3, 2, 2, 64, 100, "int8", 16)
    ws = api.Workspace(S.selkv_qcache_workspace_size(c.shape))
    k, v = rows(g, 3, 2, 60, 64, "bf16"), rows(g, 3, 2, 60, 64, "bf16")
    counts = torch.tensor([60, 40, 0], dtype=torch.int32, device="cuda")
    model = Model(c)
    api.quant_append(c, k, v, counts=counts, workspace=ws)
    model.append(k, v, [60, 40, 0])
    model.check()
    api.quant_append(c, k, v, counts=counts + 1 - (counts == 60).int(), workspace=ws)  # 60, 41, 1: the first does not fit
    assert ws.errors() == S.SELKV_DEVERR_CAPACITY
    model.append(k, v, [60, 41, 1])
    model.check()
    api.quant_append(c, k[:, :, :1].contiguous(), v[:, :, :1].contiguous(),
                     counts=torch.tensor([-1, 2, 1], dtype=torch.int32, device="cuda"), workspace=ws)
    assert ws.errors() == S.SELKV_DEVERR_LENGTH
    model.append(k[:, :, :1], v[:, :, :1], [0, 1, 1])
    model.check()
    c.lengths.copy_(torch.tensor([-3, 101, 5], dtype=torch.int32))
    api.quant_append(c, k[:, :, :1].contiguous(), v[:, :, :1].contiguous(), workspace=ws)
    assert ws.errors() == S.SELKV_DEVERR_LENGTH | S.SELKV_DEVERR_CAPACITY
    assert c.lengths.tolist() == [1, 101, 6]


# ---- reading back -----------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,d,block,cap,lens,row0,n", [
    ("bf16", 128, 64, 400, [400, 0, 131], 0, 400), ("bf16", 64, 16, 133, [133, 1, 50], 17, 101),
    ("fp32", 128, 128, 300, [299, 7, 128], 0, 300), ("fp32", 64, 32, 65, [65, 64, 2], 64, 1),
    ("bf16", 128, 32, 1100, [1100, 700, 3], 2, 1000)])
def test_read(kind, dtype, d, block, cap, lens, row0, n):
    g = gen(cap)
    B, H = len(lens), 2
    c = make(dtype, B, 4, H, d, cap, kind, block)
    k, v = rows(g, B, H, cap, d, dtype), rows(g, B, H, cap, d, dtype)
    api.quant_append(c, k, v, counts=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    model = Model(c)
    out = tuple(torch.full((B, H, n, d), 7.0, dtype=TORCH[dtype], device="cuda") for _ in range(2))
    K, V = api.quant_read(c, row0, n, out)
    assert K is out[0] and V is out[1]
    for got, side in ((K, 0), (V, 1)):
        for b in range(B):
            live = max(0, min(n, lens[b] - row0))
            for h in range(H):
                want = torch.from_numpy(model.head(b, h)[side][row0:row0 + live]).to(TORCH[dtype])
                assert torch.equal(got[b, h, :live].cpu(), want)
        at = torch.arange(n, device="cuda")[None, :] + row0 >= torch.tensor(lens, device="cuda")[:, None]
        assert bool((got.permute(0, 2, 1, 3)[at] == 7.0).all())
    whole = api.quant_read(c)[0]
    assert whole.shape == (B, H, cap, d) and torch.equal(whole[0, :, :lens[0]], api.quant_read(c, 0, lens[0])[0][0])


# ---- decode -----------------------------------------------------------------------------------------
def bound(dtype, want, pv, mag, x, n, floor):
    """How far a result may be off, from the roundings on its way, with u = 2^-24.  A logit: products of d
    terms summed in fp32 (at most (d + 8) u of sum |q k|; the sum of a chunk may be cut off instead of rounded, hence
    twice that), a query held as fp16 (bf16 queries: exactly; fp32: two halves, 2^-22), and the scale, bias and
    exponential, 8 u of the logit and 4 u.  Each p is off by as much relatively, and so is the normaliser:
    twice.  Weights rounded to fp16 (bf16 caches: 2^-11; fp32: two halves, 2^-21), a fold of n / 8 + 200
    sums, and the rounding of the output itself.
    Weights below the normal fp16 range: the kernel holds p vs (p the weight, vs the row's scale) in units of
    U 2^-10, where U is at most the largest weight of a tile of 32 rows times the largest scale of its rows.  An
    fp16 below 2^-14 is a multiple of 2^-24, so such a weight is off by at most 2^-25 units, 2^-35 U, whatever its own size.
    Times a code of at most qmax, over n rows: `floor` = n qmax 2^-35 U.  (It matters where the rows of all
    large weights hold a code 0, as int8 rows do: an element of 1e-15 next to others of 1 has no digits of its
    own.)"""
    u = 2.0 ** -24
    dlogit = 2 * (128 + 8) * u * mag + (2.0 ** -22 * mag if dtype == "fp32" else 0.0) + 8 * u * x + 4 * u
    w = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -21
    return (2 * dlogit + w + (n / 8 + 200) * u) * pv + np.abs(want) * (2.0 ** -8 if dtype == "bf16" else u) + floor + 1e-37


def check_out(c, model, out, q, app=None, k=None, v=None, use_bias=True):
    got, qs = np64(out), np64(q)
    H = model.K.shape[1]
    G = q.shape[1] // H
    dtype = "bf16" if q.dtype == torch.bfloat16 else "fp32"
    for b in range(q.shape[0]):
        for h in range(H):
            kk, vv = model.head(b, h)
            bias = model.bias[b, h, :model.L[b]] if model.bias is not None and use_bias else None
            if k is not None and app[b]:
                kk, vv = np.vstack([kk, np64(k)[b, h]]), np.vstack([vv, np64(v)[b, h]])
                bias = np.append(bias, 0.0) if bias is not None else None
            want, pv, mag, x, p = R.decode_head(qs[b, h * G:(h + 1) * G], kk, vv, bias)
            err = np.abs(got[b, h * G:(h + 1) * G] - want)
            n = int(model.L[b])
            at = np.arange(0, n, 32)
            top = np.maximum.reduceat(p[:, :n], at, 1) * np.maximum.reduceat(model.vs[b, h][np.arange(n) // model.block], at) if n else np.zeros((G, 1))
            floor = n * R.QMAX[model.kind] * 2.0 ** -35 * top.max(1)[:, None]
            lim = bound(dtype, want, pv, mag, x, kk.shape[0], floor)
            assert (err <= lim).all(), (b, h, float((err / lim).max()), float(err.max()))


def filled(dtype, B, hq, hkv, d, cap, kind, block, lens, seed, bias=True):
    g = gen(seed)
    c = make(dtype, B, hq, hkv, d, cap, kind, block, bias)
    n = max(max(lens), 1)
    k, v = rows(g, B, hkv, n, d, dtype), rows(g, B, hkv, n, d, dtype)
    bb = torch.rand((B, hkv, n), generator=g, device="cuda") if bias else None
    api.quant_append(c, k, v, bb, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    return c, g


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,B,hq,hkv,d,cap,block,lens", [
    ("bf16", 1, 8, 2, 128, 700, 64, [650]),
    ("bf16", 2, 4, 4, 128, 2100, 16, [2090, 1]),          # one query head a KV head
    ("bf16", 3, 16, 2, 64, 333, 32, [0, 331, 64]),        # eight, narrow
    ("bf16", 2, 32, 2, 128, 1030, 128, [1028, 127]),      # sixteen
    ("bf16", 2, 14, 2, 64, 200, 16, [197, 33]),           # seven
    ("bf16", 2, 22, 2, 128, 515, 128, [500, 255]),        # eleven
    ("fp32", 1, 4, 2, 64, 260, 16, [256]),
    ("fp32", 3, 8, 1, 128, 900, 64, [897, 0, 17]),
    ("fp32", 2, 16, 1, 64, 400, 128, [399, 100]),         # sixteen, fp32
    ("fp32", 2, 13, 1, 128, 190, 32, [180, 31]),          # thirteen
    ("bf16", 40, 8, 8, 128, 96, 32, [(7 * i) % 95 for i in range(40)]),
    ("bf16", 64, 16, 8, 64, 320, 64, [(37 * i) % 318 for i in range(64)]),
    ("bf16", 1, 8, 1, 128, 20000, 64, [19990]),
])
def test_decode(kind, dtype, B, hq, hkv, d, cap, block, lens):
    c, g = filled(dtype, B, hq, hkv, d, cap, kind, block, lens, hq + cap)
    model = Model(c)
    ws = api.Workspace(S.selkv_decode_q_workspace_size(c.shape))
    for token in range(3):
        q = torch.randn((B, hq, d), generator=g, device="cuda").to(TORCH[dtype])
        # queries of very different magnitude, and one of zeros
        q *= torch.tensor([1.0, 0.05, 3.0, 0.0, 1.0], device="cuda")[torch.arange(hq, device="cuda") % 5][:, None].to(q.dtype)
        k = v = None
        if token:
            k, v = (rows(g, B, hkv, 1, d, dtype)[:, :, 0].contiguous() for _ in range(2))
        app = model.L + 1 <= cap
        out = torch.full_like(q, math.nan)
        api.decode_quant(c, q, k, v, out=out, workspace=ws)
        assert ws.errors() == (0 if k is None or app.all() else S.SELKV_DEVERR_CAPACITY)
        check_out(c, model, out, q, app, k, v)
        if k is not None:
            model.append(k[:, :, None], v[:, :, None], app.astype(int))
        model.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_without_bias(dtype):
    for has in (False, True):
        c, g = filled(dtype, 2, 8, 2, 128, 300, "int8", 64, [290, 3], 9, bias=has)
        model = Model(c)
        q = torch.randn((2, 8, 128), generator=g, device="cuda").to(TORCH[dtype])
        check_out(c, model, api.decode_quant(c, q, use_bias=False), q, use_bias=False)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,hq", [("bf16", 4), ("bf16", 24), ("fp32", 4), ("fp32", 20)])
def test_decode_masks(kind, dtype, hq):
    """Bias of -inf and of the lowest finite number: on no row, some, all but one, all."""
    B, hkv, d, cap = 7, 2, 64, 500
    lens = [450, 450, 450, 450, 33, 1, 450]
    c, g = filled(dtype, B, hq, hkv, d, cap, kind, 16, lens, 3)
    low = torch.finfo(torch.float32).min
    c.bias[0, :, :450] = -math.inf
    c.bias[1, :, :450] = low
    c.bias[2, :, :450:2] = -math.inf
    c.bias[2, :, 1:450:4] = low
    c.bias[3, :, :449] = -math.inf
    c.bias[4, 0, :33] = -math.inf
    c.bias[4, 1, :33] = low
    c.bias[5, :, :1] = -math.inf
    c.bias[6, :, :450] = torch.linspace(-300, 80, 450, device="cuda")
    model = Model(c)
    q = torch.randn((B, hq, d), generator=g, device="cuda").to(TORCH[dtype])
    out = api.decode_quant(c, q)
    check_out(c, model, out, q)
    assert bool((out[0] == 0).all()) and bool((out[5] == 0).all()) and bool((out[4, :hq // 2] == 0).all())
    # with a new row: it has all the weight where the others have none
    k, v = (torch.randn((B, hkv, d), generator=g, device="cuda").to(TORCH[dtype]) for _ in range(2))
    out = api.decode_quant(c, q, k, v)
    check_out(c, model, out, q, [True] * B, k, v)
    model.append(k[:, :, None], v[:, :, None], [1] * B)
    model.check()


def test_decode_scales_far_apart():
    """Blocks whose scales differ by many orders of magnitude, some of zeros."""
    for kind in ("e4m3", "int8"):
        for dtype in ("bf16", "fp32"):
            B, hkv, d, cap, block = 1, 2, 128, 640, 16
            g = gen(11)
            c = make(dtype, B, 8, hkv, d, cap, kind, block)
            k = torch.randn((B, hkv, 600, d), generator=g, device="cuda")
            v = torch.randn((B, hkv, 600, d), generator=g, device="cuda")
            power = (torch.arange(600, device="cuda") // block * 7) % 41 - 20
            v *= (10.0 ** power)[:, None]
            v[:, :, 64:96] = 0
            k[:, :, 128:160] = 0
            k[:, :, 200:240] *= 1e-30
            k, v = k.to(TORCH[dtype]), v.to(TORCH[dtype])
            api.quant_append(c, k, v)
            q = torch.randn((B, 8, d), generator=g, device="cuda").to(TORCH[dtype])
            model = Model(c)
            check_out(c, model, api.decode_quant(c, q), q)
            # all weight on rows of tiny values: the large ones must not drown them
            c.bias[:, :, :600] = torch.where(power <= -10, 0.0, -2000.0)
            model = Model(c)
            check_out(c, model, api.decode_quant(c, q), q)


def test_decode_lengths_out_of_range():
    c, g = filled("bf16", 3, 4, 2, 64, 100, "e4m3", 32, [50, 100, 100], 4)
    ws = api.Workspace(S.selkv_decode_q_workspace_size(c.shape))
    q = torch.randn((3, 4, 64), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((3, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(2))
    model = Model(c)
    out = api.decode_quant(c, q, k, v, workspace=ws)
    assert ws.errors() == S.SELKV_DEVERR_CAPACITY
    check_out(c, model, out, q, [True, False, False], k, v)
    assert c.lengths.tolist() == [51, 100, 100]
    c.lengths.copy_(torch.tensor([-1, 101, 100], dtype=torch.int32))
    out = api.decode_quant(c, q, workspace=ws)
    assert ws.errors() == S.SELKV_DEVERR_LENGTH
    assert bool((out[0] == 0).all())
    model.L[:] = [0, 100, 100]
    check_out(c, model, out, q)


def test_decode_reads_past_32_bit_offsets():
    """A cache of more than 4 GiB of codes: its last head is read and written at its own place."""
    B, hkv, d, cap = 1, 8, 128, 4_300_000
    shape = api.make_shape("bf16", B, hkv, hkv, d, 32, cap, cap)
    c = api.alloc_quant(shape, "int8", 128)
    g = gen(8)
    k, v = rows(g, B, hkv, 300, d, "bf16"), rows(g, B, hkv, 300, d, "bf16")
    api.quant_append(c, k, v)
    model_k = c.K[0, :, :300].clone()
    q = torch.randn((B, hkv, d), generator=g, device="cuda").bfloat16()
    small = api.alloc_quant(api.make_shape("bf16", B, hkv, hkv, d, 32, 320, 320), "int8", 128)
    api.quant_append(small, k, v)
    assert torch.equal(model_k, small.K[0, :, :300])
    a, b = api.decode_quant(c, q).float(), api.decode_quant(small, q).float()
    assert float((a - b).abs().max()) <= 2.0 ** -7 * float(b.abs().max())
    # the same rows at the far end: the rows before them have no weight
    at = cap - 44
    for t, s in ((c.K, small.K), (c.V, small.V)):
        t[0, :, at - at % 128:at - at % 128 + 300 - 256] = s[0, :, 256:300]
    for t, s in ((c.K_scale, small.K_scale), (c.V_scale, small.V_scale)):
        t[0, :, at // 128] = s[0, :, 2]
        t[0, :, 3:at // 128] = 1.0
    c.bias.fill_(-math.inf)
    first = at - at % 128
    c.bias[0, :, first:first + 44] = 0.0
    c.lengths.fill_(first + 44)
    small.bias[0, :, :256] = -math.inf
    a, b = api.decode_quant(c, q).float(), api.decode_quant(small, q).float()
    assert float((a - b).abs().max()) <= 2.0 ** -7 * float(b.abs().max())
    kn, vn = rows(g, B, hkv, 1, d, "bf16"), rows(g, B, hkv, 1, d, "bf16")
    api.decode_quant(c, q, kn[:, :, 0].contiguous(), vn[:, :, 0].contiguous())
    api.quant_append(small, kn, vn)
    assert torch.equal(c.K[0, :, first + 44], small.K[0, :, 300]) and torch.equal(c.V[0, :, first + 44], small.V[0, :, 300])
    K, _ = api.quant_read(c, first, 45)
    assert torch.equal(K, api.quant_read(small, 256, 45)[0])


# ---- used together ------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind,block", [("e4m3", 64), ("int8", 32)])
def test_compress_quantise_decode_read(kind, block):
    """A prompt is compressed, its compressed cache put into 8 bits, tokens decoded over it, and the rows read
    back; the outputs stay near those over the bf16 cache."""
    g = gen(21)
    B, hq, hkv, d, n, W = 2, 8, 2, 128, 1500, 32
    K, V = (torch.randn((B, hkv, n, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    Q = torch.randn((B, hq, W, d), generator=g, device="cuda").bfloat16()
    shape = api.make_shape("bf16", B, hq, hkv, d, W, n, api.capacity(n, 0.25, 16))
    full = api.compress(shape, [n, 1201], 0.25, K, V, Q)
    c = api.quantize(full, kind, block)
    m = [375, 300]
    assert c.lengths.tolist() == m
    want = make("bf16", B, hq, hkv, d, shape.m_cap, kind, block, junk=False)
    model = Model(want)
    model.append(full.K_c, full.V_c, m, full.bias)
    model.c = c
    model.check()
    for token in range(4):
        q = torch.randn((B, hq, d), generator=g, device="cuda").bfloat16()
        k, v = (torch.randn((B, hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
        out = api.decode_quant(c, q, k, v)
        check_out(c, model, out, q, [True] * B, k, v)
        model.append(k[:, :, None], v[:, :, None], [1] * B)
        model.check()
        ref = api.decode(full, q, k, v)
        assert float((out.float() - ref.float()).norm() / ref.float().norm()) < 0.1
    K8, V8 = api.quant_read(c, 0, 379)
    for b in range(B):
        for h in range(hkv):
            kk, vv = model.head(b, h)
            assert torch.equal(K8[b, h, :m[b] + 4].cpu(), torch.from_numpy(kk).bfloat16())
            assert torch.equal(V8[b, h, :m[b] + 4].cpu(), torch.from_numpy(vv).bfloat16())


def test_tokens_in_a_captured_graph_and_on_other_streams():
    """A decode of several tokens recorded once and replayed equals the eager one; two caches at once on two
    streams, a workspace each, equal one after the other."""
    def start(seed):
        return filled("bf16", 3, 8, 2, 128, 400, "int8", 32, [200, 31, 0], seed)

    T = 6
    (a, g), (b, _) = start(1), start(1)
    q = torch.randn((T, 3, 8, 128), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((T, 3, 2, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    eager = torch.stack([api.decode_quant(a, q[t], k[t], v[t]) for t in range(T)])
    ws = api.Workspace(S.selkv_decode_q_workspace_size(b.shape))
    out = torch.empty_like(q)
    base = b.lengths.clone()
    saved = [t.clone() for t in (b.K.view(torch.int8), b.V.view(torch.int8), b.K_scale, b.V_scale)]

    def loop():
        for t in range(T):
            api.decode_quant(b, q[t], k[t], v[t], out=out[t], workspace=ws)

    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            loop()
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        b.lengths.copy_(base)
        for t, s in zip((b.K.view(torch.int8), b.V.view(torch.int8), b.K_scale, b.V_scale), saved):
            t.copy_(s)
        out.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        for x, y in ((a.K.view(torch.int8), b.K.view(torch.int8)), (a.V.view(torch.int8), b.V.view(torch.int8)),
                     (a.lengths, b.lengths)):
            assert torch.equal(x, y)
    caches = [start(s)[0] for s in (2, 3, 2, 3)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    together = [torch.empty_like(q) for _ in range(2)]
    spaces = [api.Workspace(S.selkv_decode_q_workspace_size(caches[0].shape)) for _ in range(2)]
    torch.cuda.synchronize()
    for t in range(T):
        for i in range(2):
            api.decode_quant(caches[i], q[t], k[t], v[t], out=together[i][t], workspace=spaces[i],
                             stream=streams[i] if t % 2 else streams[i].cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        alone = torch.stack([api.decode_quant(caches[2 + i], q[t], k[t], v[t]) for t in range(T)])
        assert torch.equal(together[i], alone)
        assert torch.equal(caches[i].K.view(torch.int8), caches[2 + i].K.view(torch.int8))


def test_rows_read_back_are_decoded_over_at_once():
    """selkv_qcache_read into a bf16 cache and a decode over that cache right behind it, again and again with
    other rows: the decode sees the rows of its own turn."""
    B, hq, hkv, d, cap = 1, 32, 8, 128, 9000
    shape = api.make_shape("bf16", B, hq, hkv, d, 32, cap, cap)
    g = gen(23)
    q = torch.randn((B, hq, d), generator=g, device="cuda").bfloat16()
    caches = []
    for i in range(3):
        c = api.alloc_quant(shape, "e4m3", 64)
        api.quant_append(c, rows(g, B, hkv, cap - i, d, "bf16"), rows(g, B, hkv, cap - i, d, "bf16"))
        caches.append(c)
    full = api.alloc_compressed(shape)
    ws, wr = api.Workspace(S.selkv_decode_workspace_size(shape)), api.Workspace(S.selkv_qcache_workspace_size(shape))

    def one(c, wait):
        api.quant_read(c, out=(full.K_c, full.V_c), workspace=wr)
        if wait:
            torch.cuda.synchronize()
        return api.decode(full, q, use_bias=False, workspace=ws)

    full.lengths.fill_(cap - 2)
    want = [one(c, True) for c in caches]
    assert not torch.equal(want[0], want[1])
    torch.cuda.synchronize()
    got = [one(caches[i % 3], False) for i in range(60)]
    torch.cuda.synchronize()
    assert all(torch.equal(got[i], want[i % 3]) for i in range(60))


def test_back_to_back_tokens():
    """Many tokens enqueued without a wait between them: each sees all rows before it."""
    B, hq, hkv, d, cap = 2, 8, 2, 128, 700
    c, g = filled("bf16", B, hq, hkv, d, cap, "e4m3", 64, [400, 5], 17)
    model = Model(c)
    T = 130
    q = torch.randn((T, B, hq, d), generator=g, device="cuda").bfloat16()
    # growing rows: the last block is encoded anew again and again
    size = torch.exp(torch.arange(T, device="cuda") / 40.0)[:, None, None, None]
    k, v = ((torch.randn((T, B, hkv, d), generator=g, device="cuda") * size).bfloat16() for _ in range(2))
    out = torch.empty_like(q)
    ws = api.Workspace(S.selkv_decode_q_workspace_size(c.shape))
    torch.cuda.synchronize()
    for t in range(T):
        api.decode_quant(c, q[t], k[t], v[t], out=out[t], workspace=ws)
    torch.cuda.synchronize()
    for t in range(T):
        if t % 13 == 0 or t > T - 4:
            check_out(c, model, out[t], q[t], [True] * B, k[t], v[t])
        model.append(k[t][:, :, None], v[t][:, :, None], [1] * B)
    model.check()


def test_odd_shapes_of_the_split_rule():
    """Shapes that the rule splits in each of its ways (one split, a cluster, through memory, both; CTAs of four
    and eight warps): the outputs agree with the plain form."""
    for dtype, B, hq, hkv, d, cap, n in (("bf16", 1, 4, 1, 128, 12000, 11990), ("bf16", 1, 16, 1, 128, 9000, 8000), ("fp32", 1, 2, 2, 64, 3001, 3000),
                                         ("bf16", 9, 32, 8, 64, 700, 650), ("fp32", 20, 16, 4, 128, 500, 499), ("bf16", 3, 16, 16, 128, 900, 77),
                                         ("bf16", 200, 2, 1, 64, 130, 129), ("bf16", 2, 48, 3, 128, 2600, 2500)):
        lens = [max(0, n - 37 * i % (n + 1)) for i in range(B)]
        c, g = filled(dtype, B, hq, hkv, d, cap, "int8" if cap % 2 else "e4m3", 64, lens, cap)
        model = Model(c)
        q = torch.randn((B, hq, d), generator=g, device="cuda").to(TORCH[dtype])
        k, v = (torch.randn((B, hkv, d), generator=g, device="cuda").to(TORCH[dtype]) for _ in range(2))
        out = api.decode_quant(c, q, k, v)
        check_out(c, model, out, q, [True] * B, k, v)
        model.append(k[:, :, None], v[:, :, None], [1] * B)
        model.check()


def test_the_other_sequences_outputs_do_not_depend_on_a_full_one():
    """A sequence at its capacity among others: it is not appended to, the others are, and its own output is
    that without a new row."""
    c, g = filled("bf16", 4, 8, 2, 128, 256, "int8", 32, [256, 10, 255, 0], 31)
    model = Model(c)
    q = torch.randn((4, 8, 128), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((4, 2, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    ws = api.Workspace(S.selkv_decode_q_workspace_size(c.shape))
    for turn in range(3):
        app = model.L < 256
        out = api.decode_quant(c, q, k, v, workspace=ws)
        assert ws.errors() == S.SELKV_DEVERR_CAPACITY
        check_out(c, model, out, q, app, k, v)
        model.append(k[:, :, None], v[:, :, None], app.astype(int))
        model.check()


def test_rows_without_weight_may_hold_anything():
    """Codes that are NaN, under a bias of -inf: in every tile position, for both types of K and V."""
    B, hq, hkv, d, cap = 2, 8, 2, 128, 600
    c, g = filled("bf16", B, hq, hkv, d, cap, "e4m3", 32, [590, 95], 41)
    dead = torch.rand((B, hkv, cap), generator=g, device="cuda") < 0.2
    c.bias.masked_fill_(dead, -math.inf)
    for t in (c.K, c.V):
        t.view(torch.uint8)[dead] = 0x7f
    model = Model(c)
    for t in (model.K, model.V):
        t[np.isnan(t)] = 0.0
    q = torch.randn((B, hq, d), generator=g, device="cuda").bfloat16()
    check_out(c, model, api.decode_quant(c, q), q)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,hq", [("bf16", 4), ("bf16", 24), ("fp32", 4), ("fp32", 20)])
def test_decode_halves_of_a_tile_apart(kind, dtype, hq):
    """Blocks of 16 rows, two to a tile: every other one holds values of 1e30 (or 1e12) that the bias gives no weight, or a
    weight that still counts.  The others' digits stay: the units of the weights follow the half whose weight times scale
    is the largest, so that the floor of `bound` is that of rows, not of tiles."""
    B, hkv, d, cap, n = 6, 2, 64, 640, 615
    c = make(dtype, B, hq, hkv, d, cap, kind, 16)
    g = gen(77)
    k, v = (torch.randn((B, hkv, n, d), generator=g, device="cuda") for _ in range(2))
    bias = torch.zeros((B, hkv, n), device="cuda")
    low = torch.finfo(torch.float32).min
    for b, (odd, size, weight) in enumerate([(0, 1e30, -math.inf), (1, 1e30, -math.inf), (0, 1e30, low), (1, 1e30, low),
                                             (1, 1e12, -25.0), (0, 1e-12, 20.0)]):
        at = torch.arange(n, device="cuda") // 16 % 2 == odd
        v[b, :, at] *= size
        bias[b, :, at] = weight
    v[5, :, 300:] = 0
    k, v = k.to(TORCH[dtype]), v.to(TORCH[dtype])
    api.quant_append(c, k, v, bias)
    model = Model(c)
    q = torch.randn((B, hq, d), generator=g, device="cuda").to(TORCH[dtype])
    got, qs, G = np64(api.decode_quant(c, q)), np64(q), hq // hkv
    for b in range(B):
        for h in range(hkv):
            kk, vv = model.head(b, h)
            want, pv, mag, x, p = R.decode_head(qs[b, h * G:(h + 1) * G], kk, vv, model.bias[b, h, :n])
            top = (p * model.vs[b, h][np.arange(n) // 16]).max(1)
            lim = bound(dtype, want, pv, mag, x, n, n * R.QMAX[kind] * 2.0 ** -35 * top[:, None])
            err = np.abs(got[b, h * G:(h + 1) * G] - want)
            assert (err <= lim).all(), (b, h, float((err / lim).max()))


def test_a_row_is_not_appended_without_the_bias():
    """With use_bias off a new row would leave its bias unset: refused, unless the cache has none."""
    c, g = filled("bf16", 1, 4, 2, 64, 100, "e4m3", 32, [60], 8)
    q = torch.randn((1, 4, 64), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((1, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(2))
    with pytest.raises(S.SelKVError, match="bias"):
        api.decode_quant(c, q, k, v, use_bias=False)
    model = Model(c)
    model.bias = None
    plain = api.QuantCache(c.shape, "e4m3", 32, c.K, c.V, c.K_scale, c.V_scale, None, c.lengths)
    check_out(plain, model, api.decode_quant(plain, q, k, v, use_bias=False), q, [True], k, v)
    with pytest.raises(S.SelKVError, match="workspace"):
        api.decode_quant(c, q, workspace=type("Host", (), {"buf": torch.zeros(1 << 16, dtype=torch.uint8), "nbytes": 1 << 16})())


def test_python_refusals():
    c, g = filled("bf16", 2, 8, 2, 128, 100, "e4m3", 64, [50, 3], 1)
    q = torch.zeros((2, 8, 128), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((2, 2, 128), dtype=torch.bfloat16, device="cuda")
    new = torch.zeros((2, 2, 4, 128), dtype=torch.bfloat16, device="cuda")
    n = torch.zeros((2,), dtype=torch.int32, device="cuda")
    for call in (lambda: api.decode_quant(c, q.float()), lambda: api.decode_quant(c, q[:, :4]), lambda: api.decode_quant(c, q.cpu()),
                 lambda: api.decode_quant(c, q.transpose(1, 2).contiguous().transpose(1, 2)),
                 lambda: api.decode_quant(c, q, k), lambda: api.decode_quant(c, q, None, k),
                 lambda: api.decode_quant(c, q, k, k[:, :, :64]), lambda: api.decode_quant(c, q, out=q.float()),
                 lambda: api.quant_append(c, new, new[:, :, :3]), lambda: api.quant_append(c, new[:, :, :0], new[:, :, :0]),
                 lambda: api.quant_append(c, k, k), lambda: api.quant_append(c, new, new, counts=n.long()),
                 lambda: api.quant_append(c, new, new, counts=n[:1]), lambda: api.quant_append(c, new, new, new[..., 0]),
                 lambda: api.quant_append(c, new, new, counts=c.lengths),
                 lambda: api.quant_read(c, 90, 11), lambda: api.quant_read(c, 0, 0), lambda: api.quant_read(c, -1, 4),
                 lambda: api.quant_read(c, out=(new, new.float())),
                 lambda: api.QuantCache(c.shape, "int8", 64, c.K, c.V, c.K_scale, c.V_scale, c.bias, c.lengths),
                 lambda: api.QuantCache(c.shape, "e4m3", 32, c.K, c.V, c.K_scale, c.V_scale, c.bias, c.lengths),
                 lambda: api.QuantCache(c.shape, "e4m3", 64, c.K, c.V, c.K_scale, c.V_scale, c.bias, c.lengths.long())):
        with pytest.raises(S.SelKVError):
            call()
    with pytest.raises(AttributeError):  # the tensors of a cache are not replaced
        c.bias = None
    torch.cuda.synchronize()


def test_calls_allocate_on_the_stream_they_run_on():
    """Without a workspace and outputs given, on the default stream's handle, a side stream and its handle: the same
    results, while other work allocates and frees on the current stream."""
    c, g = filled("bf16", 2, 8, 2, 128, 300, "e4m3", 32, [280, 100], 51)
    q = torch.randn((2, 8, 128), generator=g, device="cuda").bfloat16()
    want, rows_want = api.decode_quant(c, q), api.quant_read(c, 3, 200)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (0, side, side.cuda_stream):
        for _ in range(20):
            out, back = api.decode_quant(c, q, stream=stream), api.quant_read(c, 3, 200, stream=stream)
            junk = [torch.full((1 << k,), 7.0, device="cuda") for k in range(8, 20, 3)]
            del junk
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(back[0], rows_want[0]) and torch.equal(back[1], rows_want[1])
    full = api.alloc_compressed(c.shape)
    full.K_c.normal_(generator=g), full.V_c.normal_(generator=g)
    full.lengths.fill_(290)
    torch.cuda.synchronize()
    a, b = api.quantize(full, "int8", 64), api.quantize(full, "int8", 64, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(a.K, b.K) and torch.equal(a.V_scale, b.V_scale) and a.lengths.tolist() == [290, 290]
