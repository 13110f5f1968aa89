"""Plain 64-bit implementations of the operators of a speculative step, one sequence and one head at a time."""
import math

import numpy as np

MAX_TREE = 128


# ---- rotary positions ---------------------------------------------------------------------------
def frequencies(rot, theta, scaling=None, factor=1.0, original=0, low=1.0, high=32.0):
    out = []
    for f in range(rot // 2):
        w = theta ** (-2.0 * f / rot)
        if scaling is None:
            out.append(w)
            continue
        if scaling == "linear":
            keep = 0.0
        elif scaling == "wavelength":
            keep = (original * w / (2 * math.pi) - low) / (high - low)
        else:
            at = lambda n: rot * math.log(original / (2 * math.pi * n)) / (2 * math.log(theta))  # noqa: E731
            i0, i1 = max(0, math.floor(at(high))), min(rot - 1, math.ceil(at(low)))
            keep = 1.0 - (f - i0) / max(i1 - i0, 0.001)
        keep = min(1.0, max(0.0, keep))
        out.append(keep * w + (1.0 - keep) * w / factor)
    return np.array(out)


def rotate(x, pos, freq, layout, amplitude=1.0, transpose=False):
    """x [..., T, d], pos [T]; the rotation as a complex product."""
    rot = 2 * len(freq)
    y = np.array(x, dtype=np.float64)
    z = amplitude * np.exp((-1j if transpose else 1j) * np.asarray(pos, dtype=np.float64)[:, None] * freq)
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    w = (y[..., a] + 1j * y[..., b]) * z
    y[..., a], y[..., b] = w.real, w.imag
    return y


# ---- attention ----------------------------------------------------------------------------------
def ancestors(parents, n):
    """[n][n]: u is t or an ancestor of t (a parent out of range counts as none)."""
    sees = np.zeros((n, n), dtype=bool)
    for t in range(n):
        p = int(parents[t])
        sees[t, t] = True
        if 0 <= p < t:
            sees[t] |= sees[p]
    return sees


def tree_attn(q, K, V, bias, L, k_new, v_new, parents, n):
    """One sequence: q [Hq][T][d], K, V [Hkv][cap][d], bias [Hkv][cap] or None, k_new, v_new [Hkv][T][d].
    Returns out [Hq][n][d], the sums of p |v|, and each token's largest sum of |q_i k_i| / sqrt(d)."""
    Hq, _, d = q.shape
    Hkv = K.shape[0]
    sees = ancestors(parents, n)
    out, mass, size = (np.zeros((Hq, n, d)), np.zeros((Hq, n, d)), np.zeros((Hq, n, 1)))
    for h in range(Hq):
        kv = h // (Hq // Hkv)
        keep = np.ones(L, dtype=bool) if bias is None else bias[kv, :L] != -np.inf
        kk, vv = K[kv, :L][keep], V[kv, :L][keep]
        for t in range(n):
            ks = np.concatenate([kk, k_new[kv, :n][sees[t]]])
            vs = np.concatenate([vv, v_new[kv, :n][sees[t]]])
            s = ks @ q[h, t] / math.sqrt(d)
            if bias is not None:
                s[:len(kk)] += bias[kv, :L][keep]
            p = np.exp(s - s.max())
            p /= p.sum()
            out[h, t], mass[h, t] = p @ vs, p @ np.abs(vs)
            size[h, t] = (np.abs(ks) @ np.abs(q[h, t])).max() / math.sqrt(d)
    return out, mass, size


# ---- verification -------------------------------------------------------------------------------
def tree_verify(tokens, parents, uniforms, target, draft, n):
    """One sequence; arrays in 64 bits.  Returns (accepted, path, next)."""
    V = target.shape[1]
    if n == 0:
        return 0, [], -1
    node, path = 0, [0]
    while True:
        r, M, child = target[node].copy(), 1.0, -1
        for t in range(node + 1, n):
            if parents[t] != node:
                continue
            x = tokens[t]
            if draft is not None:
                if uniforms[t] * M * draft[node, x] < r[x]:
                    child = t
                    break
                rest = np.maximum(r - M * draft[node], 0.0)
                if rest.sum() > 0:
                    r, M = rest, rest.sum()
            else:
                if uniforms[t] * M < r[x]:
                    child = t
                    break
                if M - r[x] > 0:
                    M -= r[x]
                    r[x] = 0.0
        if child < 0:
            break
        node = child
        path.append(child)
    c = np.cumsum(r)
    return len(path), path, min(V - 1, int(np.searchsorted(c, uniforms[0] * c[-1], side="right")))


def random_tree(rng, T, deep=0.5):
    """Token 0 the root; another one follows the token before it with probability `deep`, else any before it."""
    return np.array([-1] + [t - 1 if rng.random() < deep else int(rng.integers(0, t)) for t in range(1, T)], dtype=np.int32)
