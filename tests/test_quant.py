"""Caches held in 8 bits on the host: the plain form against brute force, the rounding of int8 codes by
a product with the rounded reciprocal, and the refusals (no call here reaches a launch)."""
import numpy as np
import pytest
import torch

import paper_2607_16213_gb300 as S
from paper_2607_16213_gb300 import api
import quant_ref as R

FAKE = 1 << 40


@pytest.fixture(scope="module")
def lib():
    from paper_2607_16213_gb300 import build as b
    b.build()
    return S.library()


# ---- the plain form -----------------------------------------------------------------------------
def test_round_code_is_the_nearest_code():
    rng = np.random.default_rng(0)
    y = np.concatenate([rng.uniform(-460, 460, 500), rng.normal(0, 1, 500), rng.normal(0, 0.01, 500)])
    fin = np.sort(np.unique(R.E4M3[np.isfinite(R.E4M3)]))
    y = np.concatenate([y, fin, (fin[1:] + fin[:-1]) / 2])  # the codes themselves and the borders between two
    got = R.round_code(y, "e4m3")
    d = np.abs(np.clip(y, -448, 448)[:, None] - fin)
    assert np.array_equal(np.abs(got - np.clip(y, -448, 448)), d.min(1))
    ties = np.abs(d - d.min(1, keepdims=True)) == 0
    for i in np.nonzero(ties.sum(1) == 2)[0]:
        c = R.codes(got[i:i + 1], "e4m3")[0]
        assert c & 1 == 0, (y[i], got[i])
    assert np.array_equal(R.values(R.codes(got, "e4m3"), "e4m3"), got)
    t = torch.from_numpy(y).float().clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, R.round_code(y.astype(np.float32).astype(np.float64), "e4m3"))


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_fresh_scale_covers_and_is_smallest(kind):
    rng = np.random.default_rng(1)
    for A in np.concatenate([np.float32(rng.lognormal(0, 20, 300)), np.float32(R.QMAX[kind] * 2.0 ** np.arange(-20, 20))]):
        s = R.fresh_scale(float(A), kind)
        assert s * R.QMAX[kind] >= A
        m, _ = np.frexp(s)
        below = s * (0.5 if kind == "e4m3" else (m * 16 - 1) / (m * 16))
        assert s == R.MIN_SCALE or below * R.QMAX[kind] < A
        # at most an eighth of the int8 range is lost, half of the e4m3 one
        assert s == R.MIN_SCALE or A > s * R.QMAX[kind] * (0.5 if kind == "e4m3" else 8 / 9 - 1e-9)


def _fma(a, b, c):
    """fp32 fused multiply-add, by way of 64 bits (the product is exact there)."""
    return np.float32(a.astype(np.float64) * np.float64(b) + c.astype(np.float64))


def test_int8_corrected_product_rounds_as_the_quotient():
    """bf16 elements X 2^a (8 bits) over scales M/8 2^b: the fp32 product with the fp32 reciprocal, its
    remainder added back, rounds to the integer that the exact quotient rounds to, for every X, M and power
    that gives a code."""
    X = np.arange(128, 256, dtype=np.float64)
    for M in range(8, 16):
        s = np.float32(M / 8)
        rcp = np.float32(1) / s
        for a in range(-12, 1):
            x = np.float32(X * 2.0 ** a)
            exact = x.astype(np.float64) * 8  # over M
            keep = exact / M <= 127
            lo = np.floor(exact / M)
            two = 2 * exact - (2 * lo + 1) * M  # sign of quotient - (lo + 1/2), exactly
            want = np.where(two > 0, lo + 1, np.where(two < 0, lo, lo + lo % 2))
            q = x * rcp
            got = np.rint(_fma(_fma(-q, s, x), rcp, q))
            assert np.array_equal(got[keep], want[keep]), (M, a)


# ---- refusals -----------------------------------------------------------------------------------
def shape(**kw):
    base = dict(dtype=S.SELKV_BF16, batch=2, num_q_heads=32, num_kv_heads=8, head_dim=128, obs_window=64, n_cap=4096,
                m_cap=4160)
    base.update(kw)
    return S.selkv_shape(**base)


def cache(**kw):
    base = dict(type=S.SELKV_Q_E4M3, block=64, K=FAKE, V=FAKE, K_scale=FAKE, V_scale=FAKE, bias=FAKE, lengths=FAKE)
    base.update(kw)
    return S.selkv_qcache(**base)


def append(s=None, c=None, rows=5, K=FAKE, V=FAKE, bias=None, counts=None, ws=FAKE, wsb=1 << 40):
    return S.selkv_qcache_append(s or shape(), c or cache(), rows, K, V, bias, counts, ws, wsb, 0)


def read(s=None, c=None, row0=0, rows=5, K=FAKE, V=FAKE, ws=FAKE, wsb=1 << 40):
    return S.selkv_qcache_read(s or shape(), c or cache(), row0, rows, K, V, ws, wsb, 0)


def dec(s=None, c=None, q=FAKE, k=None, v=None, out=FAKE, ws=FAKE, wsb=1 << 40):
    return S.selkv_decode_attn_q(s or shape(), c or cache(), q, k, v, out, ws, wsb, 0)


@pytest.mark.parametrize("call", [append, read, dec])
def test_shared_refusals(lib, call):
    inv = S.SELKV_ERR_INVALID_ARG
    for kw in (dict(type=2), dict(type=-1), dict(block=0), dict(block=8), dict(block=48), dict(block=256), dict(K=0),
               dict(V=0), dict(K_scale=0), dict(V_scale=None), dict(lengths=0), dict(K=FAKE + 8), dict(V=FAKE + 4),
               dict(K_scale=FAKE + 4), dict(V_scale=FAKE + 8), dict(bias=FAKE + 4), dict(lengths=FAKE + 4)):
        assert call(c=cache(**kw)) == inv, kw
    for kw in (dict(dtype=2), dict(batch=0), dict(batch=1025), dict(num_kv_heads=7), dict(num_kv_heads=33, num_q_heads=33),
               dict(num_q_heads=0), dict(m_cap=0), dict(num_q_heads=17, num_kv_heads=1)):
        assert call(s=shape(**kw)) == inv, kw
    assert call(s=shape(head_dim=96)) == S.SELKV_ERR_UNSUPPORTED
    for kw in (dict(ws=0), dict(ws=FAKE + 16), dict(wsb=255)):
        assert call(**kw) == S.SELKV_ERR_WORKSPACE, kw


def test_append_refusals(lib):
    inv = S.SELKV_ERR_INVALID_ARG
    for kw in (dict(rows=0), dict(rows=-1), dict(K=0), dict(V=0), dict(K=FAKE + 8), dict(V=FAKE + 2), dict(bias=FAKE + 4),
               dict(bias=FAKE, c=cache(bias=None)), dict(counts=FAKE + 2), dict(counts=FAKE)):
        assert append(**kw) == inv, kw  # (the last: the counts are the cache's own lengths)


def test_read_refusals(lib):
    inv = S.SELKV_ERR_INVALID_ARG
    for kw in (dict(row0=-1), dict(rows=0), dict(row0=4160), dict(row0=4156), dict(rows=4161), dict(K=0), dict(V=FAKE + 8),
               dict(row0=2 ** 31 - 1, rows=2 ** 31 - 1)):
        assert read(**kw) == inv, kw


def test_decode_refusals(lib):
    inv = S.SELKV_ERR_INVALID_ARG
    for kw in (dict(q=0), dict(out=0), dict(q=FAKE + 8), dict(k=FAKE), dict(v=FAKE), dict(k=FAKE + 8, v=FAKE)):
        assert dec(**kw) == inv, kw
    assert dec(s=shape(batch=1024, num_kv_heads=32, m_cap=65536)) == S.SELKV_ERR_UNSUPPORTED


def test_workspace_sizes(lib):
    assert S.selkv_qcache_workspace_size(shape()) == 512
    assert S.selkv_decode_q_workspace_size(shape()) > 512
    for f in (S.selkv_qcache_workspace_size, S.selkv_decode_q_workspace_size):
        assert f(shape(batch=0)) == 0 and f(shape(num_kv_heads=7)) == 0
    need = S.selkv_decode_q_workspace_size(shape())
    assert dec(wsb=need - 1) == S.SELKV_ERR_WORKSPACE
    assert append(wsb=511) == S.SELKV_ERR_WORKSPACE and read(wsb=511) == S.SELKV_ERR_WORKSPACE


def test_python_refusals_on_the_host():
    s = api.make_shape("bf16", 1, 4, 2, 64, 8, 64, 64)
    with pytest.raises(S.SelKVError):
        api.alloc_quant(s, "e5m2", 64, device="cpu")
    with pytest.raises(S.SelKVError):
        api.alloc_quant(s, "int8", 24, device="cpu")
    with pytest.raises(S.SelKVError, match="CUDA"):  # a cache lives on a GPU
        api.alloc_quant(s, "int8", 64, device="cpu")


def test_rows_out_of_range(lib):
    """No rows, and more than are counted in 32 bits: a size of 0 and refusals."""
    for m_cap in (0, 2 ** 30 + 1, 2 ** 31 - 1):
        s = shape(batch=1, num_q_heads=4, num_kv_heads=1, m_cap=m_cap)
        assert S.selkv_decode_q_workspace_size(s) == 0
        want = S.SELKV_ERR_INVALID_ARG if m_cap == 0 else S.SELKV_ERR_UNSUPPORTED
        assert append(s=s) == want and read(s=s) == want and dec(s=s) == want
    assert S.selkv_decode_q_workspace_size(shape(head_dim=96)) == 0
    assert S.selkv_decode_q_workspace_size(shape(batch=1, num_q_heads=4, num_kv_heads=1, m_cap=2 ** 30)) > 0
    assert append(rows=2 ** 30 + 1) == S.SELKV_ERR_UNSUPPORTED


def test_counts_overlap_the_lengths(lib):
    """Counts that share some of their bytes with the cache's own lengths (two sequences)."""
    for at in (-4, 0, 4):
        assert append(s=shape(batch=2), c=cache(lengths=FAKE), counts=FAKE + at) == S.SELKV_ERR_INVALID_ARG
    # (beside them they are taken: the next check refuses)
    for at in (-8, 8):
        assert append(s=shape(batch=2), c=cache(lengths=FAKE), counts=FAKE + at, ws=0) == S.SELKV_ERR_WORKSPACE
