"""Caches held in 8 bits at their edges, against the plain form in 64 bits: workspaces that go from one cache to
another."""
import math

import pytest
import torch

import paper_2607_16213_gb300 as S
from paper_2607_16213_gb300 import api
from test_gpu_quant import Model, filled, gen, rows

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
