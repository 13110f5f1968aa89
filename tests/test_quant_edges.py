"""Caches held in 8 bits on the host, at their edges."""
import pytest

import paper_2607_16213_gb300 as S


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
