"""Caches held in 8 bits, in plain numpy and 64 bits: scales, codes, append, read and decode by their
definitions (include/selkv.h), with explicit loops over blocks.  A cache here holds the values of the
codes (without their scale) as float64."""
import math

import numpy as np

QMAX = {"e4m3": 448.0, "int8": 127.0}
MIN_SCALE = 2.0 ** -100


def e4m3_values():
    """Value of each of the 256 e4m3 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinities."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        out[c] = math.nan if c & 127 == 127 else (-v if c & 128 else v)
    return out


E4M3 = e4m3_values()


def values(codes_u8, kind):
    return E4M3[codes_u8] if kind == "e4m3" else codes_u8.view(np.int8).astype(np.float64)


def codes(v, kind):
    """The bytes of code values (for int8 and finite e4m3 values)."""
    if kind == "int8":
        return v.astype(np.int8).view(np.uint8)
    pos = E4M3[:127]
    c = np.searchsorted(pos, np.abs(v)).astype(np.uint8)
    return c | np.where(np.signbit(v), 128, 0).astype(np.uint8)


def round_code(y, kind):
    """y to the nearest value that a code has, ties to even, infinities to the largest."""
    q = QMAX[kind]
    y = np.clip(y, -q, q)
    if kind == "int8":
        return np.where(np.isnan(y), 0.0, np.rint(y))
    a = np.abs(y)
    _, e = np.frexp(np.maximum(np.nan_to_num(a), 2.0 ** -6))
    step = np.ldexp(1.0, e - 4)
    return np.rint(y / step) * step


def fresh_scale(A, kind):
    """Smallest s of the grid with s * qmax >= A, by going up the grid."""
    ms = [1.0] if kind == "e4m3" else [m / 8 for m in range(8, 16)]
    if A <= MIN_SCALE * QMAX[kind]:
        return MIN_SCALE
    e = math.floor(math.log2(A / QMAX[kind])) - 2
    while True:
        for m in ms:
            s = m * 2.0 ** e
            if s * QMAX[kind] >= A:
                return s
        e += 1


def grown_scale(s0, A, kind):
    s = max(s0, MIN_SCALE)
    while s * QMAX[kind] < A:
        s *= 2
    return s


def append_head(val, scale, x, L, block, kind):
    """Rows x [n][d] behind the first L of val [cap][d] (in place); scale [blocks]."""
    n = x.shape[0]
    if n == 0:
        return
    fin = np.where(np.isfinite(x), np.abs(x), 0.0)
    for p in range(L // block, -(-(L + n) // block)):
        r0, r1 = max(L, p * block), min(L + n, (p + 1) * block)
        A = fin[r0 - L:r1 - L].max()
        if r0 > p * block:
            s = grown_scale(scale[p], A, kind)
            s0 = max(scale[p], MIN_SCALE)
            if s != s0:
                val[p * block:r0] = round_code(val[p * block:r0] * (s0 / s), kind)
        else:
            s = fresh_scale(A, kind)
        scale[p] = s
        val[r0:r1] = round_code(x[r0 - L:r1 - L] / s, kind)


def decode_head(q, k, v, bias):
    """q [G][d], k, v [n][d], bias [n] or None -> (out [G][d], sum p|v|, the largest sum_j |q_j k_j| / sqrt(d) and |logit|, p)."""
    G, d = q.shape
    if k.shape[0] == 0:
        return np.zeros((G, d)), np.zeros((G, d)), 0.0, 0.0, np.zeros((G, 0))
    s = q @ k.T / math.sqrt(d)
    mag = (np.abs(q) @ np.abs(k).T / math.sqrt(d)).max()
    if bias is not None:
        s = s + bias
    m = s.max(1, keepdims=True)
    live = m > -math.inf
    p = np.exp(s - np.where(live, m, 0.0))
    z = p.sum(1, keepdims=True)
    p = p / np.where(z > 0, z, 1.0)
    fin = np.abs(s[np.isfinite(s)])
    return p @ v, p @ np.abs(v), mag, (fin[fin < 1e30].max() if (fin < 1e30).any() else 0.0), p
