"""The kernels that accumulate attention weights, without time to wait: an error code, nothing written outside, and the context stays usable."""
import pytest
import torch

import paper_2505_21467_b200 as dlm
import q4_reference as ref
from helpers import Dev
from test_gpu_cache_evict import Plain, accumulate
from test_gpu_cache_q4 import Cache, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return Dev()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", [Cache, Plain])
@pytest.mark.parametrize("g,L,C", [(1, 1, 100), (7, 32, 1500), (5, 77, 700)], ids=["one_tile", "rows_that_stay", "rows_that_go_through"])
def test_the_kernels_give_up_instead_of_hanging(dev, kind, D, g, L, C):
    NL, H, capacity = 4, 8, (C + 15) // 8 * 8
    c = kind(dev, NL, 1, H, capacity, D, [C], 701)
    q, kn, vn = inputs(NL, 1, g * H, H, L, D, [L], 702)
    lse = torch.full((NL, 1, g * H, L), 8.0)
    weight = dev.guarded((NL, 1, H, capacity), torch.float32, 3.0)
    dlm.dlm_selftest_set_wait_limit(dev.ctx, 0)
    try:
        accumulate(dev, c, q.cuda(), lse.cuda(), None, weight, 0.5, weight)
        assert dev.status() == dlm.DLM_ERR_TIMEOUT
    finally:
        dlm.dlm_selftest_set_wait_limit(dev.ctx, 2_000_000_000)
    assert bool((weight[..., C:] == 3.0).all())
    weight = dev.guarded((NL, 1, H, capacity), torch.float32, 3.0)
    accumulate(dev, c, q.cuda(), lse.cuda(), None, weight, 0.5, weight)
    assert dev.status() == 0
    want, most = ref.weights(c.values("k", NL - 1), [C], q[NL - 1], lse[NL - 1], [L], torch.full((1, H, capacity), 3.0), 0.5)
    rel = 2 * D * 2.0 ** -24 * most + 2.0 ** -22 * most + 2.0 ** -20 + g * L * 2.0 ** -24      # as test_weights_match_64_bits has it
    seen = ~want.isnan()
    assert bool(((weight[NL - 1].cpu().double() - want).abs() <= rel * want + 2.0 ** -22)[seen].all())
