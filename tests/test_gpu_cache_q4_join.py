"""The join of split units finds its parts from the lengths: which may have been written by whatever ran right before the attention call."""
import pytest
import torch

import paper_2505_21467_b200 as dlm
from helpers import Dev
from test_gpu_cache_q4 import Cache, check_attention, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return Dev()


@pytest.mark.parametrize("D,g,L", [(128, 7, 32), (128, 1, 3), (64, 2, 40), (64, 3, 10)])
def test_lengths_that_change_from_call_to_call(dev, D, g, L):
    """Calls without a pause, each behind a copy that sets both lengths anew, so that units are split at other places every time; with a pause between
    them the same bits, and what 64 bits say."""
    B, H, capacity = 3, 2, 2048
    lens = [[2000, 5, 700], [0, 0, 2048], [1, 1999, 64], [300, 300, 300], [2048, 2048, 2048], [64, 0, 1], [0, 2000, 0], [1300, 17, 1301]]
    rows = [[L, L, 1], [L, 0, L], [1, L, L], [L, L, L], [L, 1, L], [L, L, L], [0, L, L], [L, L, 2]]
    c = Cache(dev, 1, B, H, capacity, D, [capacity] * B, 601)
    q, kn, vn = inputs(1, B, g * H, H, L, D, [L] * B, 602)
    gq, gk, gv = q.cuda(), kn.cuda(), vn.cuda()
    at, lq = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in (lens, rows))
    q_len = lq[0].clone()
    ws = dev.guarded((dlm.dlm_attn_workspace_bytes_q4(dev.ctx, c.view, 1, g * H, L),), torch.uint8, 0)
    results = []
    for pause in (False, True):
        outs = []
        torch.cuda.synchronize()
        for i in range(len(lens)):
            out, lse = torch.empty_like(gq), torch.empty(1, B, g * H, L, device="cuda")
            c.cache_len.copy_(at[i])
            q_len.copy_(lq[i])
            dlm.dlm_freecache_attn_step_q4(dev.ctx, c.view, 0, 1, gq, gk, gv, g * H, L, q_len, 0.0, 0, out, lse, ws)
            if pause:
                torch.cuda.synchronize()
            outs.append((out, lse))
        assert dev.status() == 0
        results.append(outs)
        ws = dev.guarded(tuple(ws.shape), torch.uint8, 255)
    for i, (one, two) in enumerate(zip(*results)):
        assert torch.equal(one[0].view(torch.int16), two[0].view(torch.int16)) and torch.equal(one[1], two[1]), i
        c.cache_len.copy_(at[i])
        check_attention(c, q, kn, vn, rows[i], *one)
