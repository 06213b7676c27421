"""What the calls on a 4-bit cache promise of rows and counts out of range, and that they stay within their workspace."""
import pytest
import torch

import paper_2505_21467_b200 as dlm
import q4_reference as ref
from helpers import Dev
from test_gpu_cache_q4 import Cache, check_attention, hard_rows, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return Dev()


def read(dev, c, pos, n_rows, n_max, lb, le):
    NL, B, H, capacity, D = c.shape
    out = [dev.guarded((le - lb, B, H, n_max, D), torch.bfloat16, 3.0) for _ in range(2)]
    dlm.dlm_kv_cache_read_q4(dev.ctx, c.view, pos.cuda(), None if n_rows is None else n_rows.cuda(), n_max, lb, le, *out)
    return out


def expected(c, name, pos, counts, n_max, lb, le):
    NL, B, H, capacity, D = c.shape
    want = torch.full((le - lb, B, H, n_max, D), 3.0, dtype=torch.float64)
    for l in range(lb, le):
        val = c.values(name, l)
        for b in range(B):
            for r in range(counts[b]):
                if 0 <= pos[b, r] < capacity:
                    want[l - lb, b, :, r] = val[b][:, int(pos[b, r])]
    return want


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("wrong", [-1, 72, 1 << 30, -(1 << 31)])
def test_a_position_out_of_range_skips_that_row_alone(dev, D, wrong):
    c = Cache(dev, 3, 2, 2, 72, D, [11, 40], 801)
    pos = torch.randint(0, 72, (2, 9), generator=torch.Generator().manual_seed(802)).int()
    for b, r in ((0, 0), (1, 8), (1, 3)):
        bad = pos.clone()
        bad[b, r] = wrong
        ko, vo = read(dev, c, bad, None, 9, 1, 3)
        assert dev.status() == dlm.DLM_ERR_INDEX
        for name, got in (("k", ko), ("v", vo)):
            assert torch.equal(got.cpu().double(), expected(c, name, bad, [9, 9], 9, 1, 3))
    ko, vo = read(dev, c, pos, None, 9, 0, 3)                          # and the next call has no error
    assert dev.status() == 0
    assert torch.equal(ko.cpu().double(), expected(c, "k", pos, [9, 9], 9, 0, 3))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("wrong", [-1, 10, 1 << 30])
def test_a_count_out_of_range_writes_nothing_for_that_sequence(dev, D, wrong):
    c = Cache(dev, 2, 3, 2, 72, D, [11, 40, 0], 811)
    pos = torch.randint(0, 72, (3, 9), generator=torch.Generator().manual_seed(812)).int()
    ko, vo = read(dev, c, pos, torch.tensor([4, wrong, 9], dtype=torch.int32), 9, 0, 2)
    assert dev.status() == dlm.DLM_ERR_CAPACITY
    for name, got in (("k", ko), ("v", vo)):
        assert torch.equal(got.cpu().double(), expected(c, name, pos, [4, 0, 9], 9, 0, 2))
    pos[2, 8], pos[0, 4] = 72, -5                                      # only rows that are read count
    ko, vo = read(dev, c, pos, torch.tensor([4, 0, 8], dtype=torch.int32), 9, 0, 2)
    assert dev.status() == 0
    assert torch.equal(vo.cpu().double(), expected(c, "v", pos, [4, 0, 8], 9, 0, 2))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 300])
def test_counts_out_of_range_commit_nothing_for_that_sequence(dev, D, n):
    c = Cache(dev, 2, 3, 4, 400, D, [11, 40, 0], 821)
    g = torch.Generator().manual_seed(822)
    k, v = hard_rows(g, 2, 3, 4, n, D), hard_rows(g, 2, 3, 4, n, D)
    for wrong in (-1, n + 1):
        c.cache_len.copy_(torch.tensor([11, 40, 0]))
        dlm.dlm_kv_cache_commit_q4(dev.ctx, c.view, k.cuda(), v.cuda(), n, None, None, dlm.DLM_DST_APPEND, torch.tensor([n, wrong, n], dtype=torch.int32).cuda(), n, 1, 0, 2)
        assert dev.status() == dlm.DLM_ERR_CAPACITY
        for name, t in (("k", k), ("v", v)):
            data, scale = ref.pack(*ref.quantise(t))
            for b, at in ((0, 11), (2, 0)):
                c.host[name][:, b, :, at:at + n], c.host[name + "_scale"][:, b, :, at:at + n] = data[:, b], scale[:, b]
        c.check_bytes()
        assert c.cache_len.tolist() == [11 + n, 40, n]


# every kernel of the attention, with units that are split over many blocks: parts fill the workspace
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("NL,B,g,L,C", [(1, 1, 1, 1, 9000), (1, 1, 1, 16, 9000), (1, 1, 2, 16, 9000), (1, 1, 3, 11, 9000), (1, 1, 2, 64, 6000), (1, 1, 7, 32, 6000),
                                        (1, 1, 3, 171, 2000), (7, 3, 1, 5, 1504), (7, 3, 5, 40, 704)])
def test_parts_stay_within_the_workspace(dev, D, NL, B, g, L, C):
    """The workspace is as large as dlm_attn_workspace_bytes_q4 says, to the byte, between guards, and holds NaN to begin with."""
    lens = [C - 100 * b for b in range(B)]
    c = Cache(dev, NL, B, 2, C, D, lens, 831)
    q, kn, vn = inputs(NL, B, 2 * g, 2, L, D, [L] * B, 832)
    n = dlm.dlm_attn_workspace_bytes_q4(dev.ctx, c.view, NL, 2 * g, L)
    ws = dev.guarded((n,), torch.uint8, 255)
    out, lse = dev.guarded(tuple(q.shape), torch.bfloat16, float("nan")), dev.guarded(tuple(q.shape[:4]), torch.float32, float("nan"))
    dlm.dlm_freecache_attn_step_q4(dev.ctx, c.view, 0, NL, q.cuda(), kn.cuda(), vn.cuda(), 2 * g, L, None, 0.0, 0, out, lse, ws)
    assert dev.status() == 0
    check_attention(c, q, kn, vn, [L] * B, out, lse)
