"""Sizes and types that the host turns away: the workspace of a call that the attention over a 4-bit cache refuses, and views of other types."""
import ctypes

import pytest
import torch

import paper_2505_21467_b200 as dlm
from paper_2505_21467_b200 import build as _build


@pytest.fixture(scope="module", autouse=True)
def built():
    _build.build()


def _workspace_bytes(cache, layers, heads, q_cap, sms=148):
    ctx = (ctypes.c_int32 * 4096)(0, sms)      # stands for a context: its second word is the number of SMs
    return dlm.dlm_attn_workspace_bytes_q4(ctypes.addressof(ctx), cache, layers, heads, q_cap)


def _cache(**kw):
    a = dict(k=None, v=None, k_scale=None, v_scale=None, cache_len=None, n_layers=2, batch=2, n_kv_heads=2, capacity=64, head_dim=64)
    a.update(kw)
    return dlm.dlm_kv_cache_q4(*a.values())


def test_workspace_holds_two_parts_a_block():
    """Output, maximum and sum in fp32 of the rows of a unit (at most 256, in whole warps), twice for each SM."""
    for D in (64, 128):
        for heads, q_cap, rows in ((2, 1, 32), (4, 40, 96), (14, 32, 224), (2, 256, 256), (64, 4096, 256)):
            assert _workspace_bytes(_cache(head_dim=D), 1, heads, q_cap) == 2 * 148 * rows * (D + 2) * 4


def test_workspace_of_calls_that_are_refused_is_zero():
    for c, args in ((_cache(), (0, 4, 8)), (_cache(), (1, 3, 8)), (_cache(), (1, 0, 8)), (_cache(), (1, 4, 0)), (_cache(), (1, 4, 4097)), (_cache(head_dim=96), (1, 4, 8)),
                    (_cache(n_kv_heads=0), (1, 4, 8)), (_cache(batch=0), (1, 4, 8))):
        assert _workspace_bytes(c, *args) == 0, args
    # more than 2^20 query rows a KV head, past 32 bits too; more than 1024 sequences
    for c, args in ((_cache(n_kv_heads=1), (1, 257, 4096)), (_cache(n_kv_heads=1), (1, 1 << 19, 4096)), (_cache(n_kv_heads=1), (1, (1 << 31) - 1, 4096)),
                    (_cache(n_kv_heads=1), (1, 1 << 20, 4096)), (_cache(batch=1025), (1, 4, 8))):
        assert _workspace_bytes(c, *args) == 0, args
    assert _workspace_bytes(_cache(n_kv_heads=1, batch=1024), 1, 256, 4096) > 0

def test_views_take_bytes_only():
    data, scale, n = torch.zeros(1, 2, 2, 8, 32, dtype=torch.uint8), torch.zeros(1, 2, 2, 8, 2, dtype=torch.uint8), torch.zeros(2, dtype=torch.int32)
    for v in (data.to(torch.bfloat16), data.to(torch.int8), data.float()):
        with pytest.raises(TypeError, match="k and v must be uint8"):
            dlm.make_kv_cache_q4(data, v, scale, scale, n)
    for v_scale in (scale.float(), scale.to(torch.int8)):
        with pytest.raises(TypeError, match="k_scale and v_scale must be uint8"):
            dlm.make_kv_cache_q4(data, data, scale, v_scale, n)
