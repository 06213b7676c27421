"""Two programs' calls at once: a context, a stream and buffers each."""
import pytest
import torch

import paper_2505_21467_b200 as dlm
from helpers import Dev
from test_gpu_cache_q4 import Cache, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g,L", [(1, 3), (2, 20), (7, 24)])
def test_two_loops_beside_each_other(D, g, L):
    """Attention, weights, commit and eviction on two streams without a pause: the same bits as one loop after the other."""
    NL, B, H, capacity, keep = 4, 3, 4, 480, 400
    devs = [Dev(), Dev()]
    steps = [[[t.cuda() for t in inputs(NL, B, g * H, H, L, D, [L] * B, 1000 * p + i)] for i in range(6)] for p in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    for together in (False, True):
        progs = []
        for p, dev in enumerate(devs):
            c = Cache(dev, NL, B, H, capacity, D, [390, 17, 0], 1100 + p)
            ws = torch.empty(dlm.dlm_attn_workspace_bytes_q4(dev.ctx, c.view, NL, g * H, L), dtype=torch.uint8, device="cuda")
            progs.append(dict(dev=dev, c=c, ws=ws, weight=torch.zeros(NL, B, H, capacity, device="cuda"),
                              kept=torch.empty(NL, B, H, keep, dtype=torch.int32, device="cuda"),
                              out=[torch.empty_like(s[0]) for s in steps[p]], lse=[torch.empty(NL, B, g * H, L, device="cuda") for _ in steps[p]]))
        torch.cuda.synchronize()

        def step(p, i):
            s, (q, kn, vn) = progs[p], steps[p][i]
            ctx, view, w = s["dev"].ctx, s["c"].view, s["weight"]
            dlm.dlm_freecache_attn_step_q4(ctx, view, 0, NL, q, kn, vn, g * H, L, None, 0.0, 0, s["out"][i], s["lse"][i], s["ws"])
            dlm.dlm_cache_weight_accumulate_q4(ctx, view, 0, NL, q, s["lse"][i], g * H, L, None, 0.0, 0, w, 0.9, w)
            dlm.dlm_kv_cache_commit_q4(ctx, view, kn, vn, L, None, None, dlm.DLM_DST_APPEND, None, L, 1, 0, NL)
            dlm.dlm_kv_cache_evict_q4(ctx, view, w, keep, 2, L, s["kept"], w)

        if together:
            for i in range(6):
                for p in range(2):
                    with torch.cuda.stream(streams[p]):
                        step(p, i)
        else:
            for p in range(2):
                for i in range(6):
                    step(p, i)
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert [dev.status() for dev in devs] == [0, 0]
        results.append([t.clone() for s in progs for t in (*s["out"], *s["lse"], s["weight"], s["kept"], s["c"].cache_len, *s["c"].gpu.values())])
    for one, two in zip(*results):
        assert torch.equal(one.view(torch.uint8), two.view(torch.uint8))
