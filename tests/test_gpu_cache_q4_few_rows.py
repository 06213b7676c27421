"""Attention over the 4-bit cache for few query rows a KV head: parts of a single tile of keys, which one of a block's two groups computes and both
read, next to parts of many."""
import pytest
import torch

import q4_reference as ref
from helpers import Dev
from test_gpu_cache_q4 import Cache, attention_call, check_attention, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return Dev()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g,L", [(1, 1), (1, 9), (4, 4), (3, 7), (8, 4)])
@pytest.mark.parametrize("lens", [[0, 0, 0], [0, 130, 0], [1, 0, 900]], ids=str)
def test_units_of_one_tile_next_to_longer_ones(dev, D, g, L, lens):
    """With an empty cache a unit is the fresh rows' tile alone.  More units than blocks, so that a block's parts of one tile and of several follow each
    other and their outputs lie in the same columns.  The same bits every time."""
    NL, H, lq = 8, 8, [L, L, max(1, L - 1)]
    c = Cache(dev, NL, 3, H, (max(lens) + 8) // 8 * 8, D, lens, 501)
    q, kn, vn = inputs(NL, 3, g * H, H, L, D, lq, 502)
    q_len = torch.tensor(lq, dtype=torch.int32, device="cuda")
    first = None
    for _ in range(4):
        out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), q_len)
        assert dev.status() == 0
        if first is None:
            first = out, lse
            check_attention(c, q, kn, vn, lq, out, lse)
        assert torch.equal(out.view(torch.int16), first[0].view(torch.int16)) and torch.equal(lse, first[1])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g,L", [(1, 2), (2, 13)])
def test_references_that_move_in_every_tile(dev, D, g, L):
    """Keys whose scores rise from tile to tile by more than the references allow: O^T and the sums are moved each time, in both groups, and what
    the last tile leaves is what 64 bits say."""
    C = 1280
    c = Cache(dev, 2, 1, 2, C, D, [C], 511)
    k = torch.randn(2, 1, 2, C, D, generator=torch.Generator().manual_seed(512)) * 0.05
    k[..., 0] = torch.arange(C).div(128, rounding_mode="floor") * 400.0      # 400 q0 D^-0.5: 35 units and more a tile
    c.host["k"], c.host["k_scale"] = ref.pack(*ref.quantise(k.bfloat16()))
    c.gpu["k"].copy_(c.host["k"]), c.gpu["k_scale"].copy_(c.host["k_scale"])
    q, kn, vn = inputs(2, 1, 2 * g, 2, L, D, [L], 513)
    q[..., 0] = q[..., 0].abs() + 1
    kn[..., 0] = 0
    out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None)
    assert dev.status() == 0
    check_attention(c, q, kn, vn, [L], out, lse)
