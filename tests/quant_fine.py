"""Small decodes over fp32 8-bit caches on which every half counts: inputs, the 64-bit result, how far a result may be off, and the
mistakes of holding queries or weights in one half (on the host).

Roundings, with u = 2^-24, s_i = q . k_i / sqrt(d) and R_i = sqrt(sum_j (q_j k_ij)^2 / d) (what independent errors of the products
add up to).  Relative errors of a weight p_i that are independent between rows, in square mean:
  - a query element as two halves is off by at most 2^-22 of itself: 2^-22 R_i;
  - each of the d / 16 steps of a sum on the tensor cores adds 16 products to the sum so far and cuts all 17 off at 2^-23 of
    the largest of them or lower; partial sums and products are below 4 R_i sqrt(d) but for one in ten thousand:
    sqrt(17 d / 16) 2^-21 R_i.
Errors that may have one sign for all rows: cut-off sums shrink by 2^-23 a step, (d / 16 + 1) 2^-23 |s_i|; the factor, the
bias and the difference to the largest logit, 8 u of the largest |logit| of the row's head; the exponential 4 u, the weight as
two halves 4 u.  An error e_i of p_i moves the output by p_i (v_i - out) e_i.  The sums behind: sixteen products and a sum cut off at
2^-23 of the largest, twice for a tile's half, independent: sqrt(34 n / 16) 2^-23 max_i |p_i v_i|; adding the halves of tiles,
warps and splits, n / 16 + 20 roundings of partial sums of at most sum_i p_i |v_i|, twice (output and normaliser).  Weights
below the normal fp16 range: n 2^-33 max|v| max p.  The independent parts count six times their square mean."""
import math

import numpy as np

import quant_ref as R

# d, query heads, KV heads, rows of each sequence, type, block
CASES = [
    (128, 4, 2, [40, 17], "int8", 16),
    (64, 16, 2, [96, 33, 64], "e4m3", 64),
    (128, 12, 1, [33, 100], "int8", 128),
    (64, 16, 1, [200, 48], "e4m3", 16),
    (128, 8, 2, [600], "int8", 32),
]


def inputs(case, seed):
    """q [B][Hq][d], k and v [B][Hkv][n][d], bias [B][Hkv][n], fp32: unit rows and queries."""
    d, hq, hkv, lens, _, _ = case
    rng = np.random.default_rng(seed)
    n, B = max(lens), len(lens)
    f = lambda *s: rng.standard_normal(s).astype(np.float32)
    return f(B, hq, d), f(B, hkv, n, d), f(B, hkv, n, d), rng.random((B, hkv, n)).astype(np.float32)


def cached(x, n, kind, block):
    """What an 8-bit cache holds of rows x [n][d]: the values, and the scale of each row."""
    val, scale = np.zeros_like(x, dtype=np.float64), np.zeros(-(-n // block))
    R.append_head(val, scale, x.astype(np.float64)[:n], 0, block, kind)
    s = scale[np.arange(n) // block]
    return val[:n] * s[:, None], s


def limit(q, k, v, bias):
    """(out, how far a result may be off) for q [G][d], k and v [n][d]."""
    u, (n, d) = 2.0 ** -24, k.shape
    out, _, _, _, p = R.decode_head(q, k, v, bias)
    s = q @ k.T / math.sqrt(d)
    r = np.sqrt((q ** 2) @ (k ** 2).T / d)
    alone = (2.0 ** -22 + math.sqrt(17 * d / 16) * 2.0 ** -21) * r
    shared = (d / 16 + 1) * 2.0 ** -23 * np.abs(s) + 8 * u * np.abs(s + bias).max(1, keepdims=True) + 8 * u
    far = np.abs(v[None] - out[:, None])  # [G][n][d]
    lim = 6 * np.sqrt(((p * alone)[..., None] ** 2 * far ** 2).sum(1)) + ((p * shared)[..., None] * far).sum(1)
    pv = p[..., None] * np.abs(v)[None]
    lim += 6 * math.sqrt(34 * n / 16) * 2.0 ** -23 * pv.max(1) + 2 * (n / 16 + 20) * u * pv.sum(1)
    return out, lim + n * 2.0 ** -33 * np.abs(v).max() * p.max(1, keepdims=True) + u * np.abs(out)


def halves(x, parts):
    """x held as one or two halves, scaled by a power of two to a largest magnitude in [2^14, 2^15) first."""
    up = 2.0 ** (14 - math.floor(math.log2(np.abs(x).max())))
    a = np.float16(x * up).astype(np.float64)
    return (a + (np.float16(x * up - a).astype(np.float64) if parts == 2 else 0)) / up


def emulated(q, k, v, bias, scale, q_parts, p_parts):
    """The decode with queries and weights times the V scale held in one or two halves, all else in 64 bits."""
    s = np.stack([halves(x, q_parts) for x in q]) @ k.T / math.sqrt(k.shape[1]) + bias
    p = np.exp(s - s.max(1, keepdims=True))
    w = np.stack([halves(x, p_parts) for x in p * scale])
    return w @ (v / scale[:, None]) / p.sum(1, keepdims=True)
