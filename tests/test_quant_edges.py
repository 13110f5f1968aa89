"""Caches held in 8 bits on the host, at their edges."""
import numpy as np
import pytest

import paper_2607_16213_gb300 as S
import quant_fine as F


@pytest.fixture(scope="module")
def lib():
    from paper_2607_16213_gb300 import build as b
    b.build()
    return S.library()


def test_decode_counters_lie_at_one_place(lib):
    """A decode without partials needs as much for every batch, dtype and group: what its counters take does not depend on the
    shape, so that those of the next cache on a workspace never lie where this one's partials were."""
    sizes = {S.selkv_decode_q_workspace_size(S.selkv_shape(dtype, batch, hkv * G, hkv, d, 64, 64, 64))
             for dtype in (S.SELKV_BF16, S.SELKV_FP32) for batch in (1, 64, 1024) for hkv in (1, 32) for G in (1, 16) for d in (64, 128)}
    assert len(sizes) == 1
    assert sizes.pop() >= S.selkv_qcache_workspace_size(S.selkv_shape(S.SELKV_BF16, 1024, 32, 32, 128, 64, 64, 64))


@pytest.mark.parametrize("case", F.CASES)
def test_the_fine_limit_tells_one_half_from_two(case):
    """The limit that fp32 decodes are held to: queries and weights in two halves stay well below it, either of them in one
    half goes past it."""
    d, hq, hkv, lens, kind, block = case
    q, k, v, bias = (x.astype(np.float64) for x in F.inputs(case, 1))
    worst = {}
    for b, n in enumerate(lens):
        for h in range(hkv):
            G = hq // hkv
            qs, (kk, _), (vv, scale) = q[b, h * G:(h + 1) * G], F.cached(k[b, h], n, kind, block), F.cached(v[b, h], n, kind, block)
            out, lim = F.limit(qs, kk, vv, bias[b, h, :n])
            for parts in ((2, 2), (1, 2), (2, 1)):
                err = np.abs(F.emulated(qs, kk, vv, bias[b, h, :n], scale, *parts) - out)
                worst[parts] = max(worst.get(parts, 0.0), float((err / lim).max()))
    assert worst[2, 2] < 0.25 and worst[1, 2] > 2 and worst[2, 1] > 2, worst
