"""The 4-bit rows' definition, and the argument checks of the calls on a 4-bit cache, on attention weights and on eviction (no GPU needed: an
argument error is returned before anything is launched or any device pointer is read)."""
import ctypes

import pytest
import torch

import paper_2505_21467_b200 as dlm
import q4_reference as ref
from paper_2505_21467_b200 import build as _build


@pytest.fixture(scope="module", autouse=True)
def built():
    _build.build()


def test_scales_are_exact_in_bf16_with_their_values():
    for b in range(256):
        bits = ((b << 4) + (107 << 7)) << 16
        assert torch.tensor(bits, dtype=torch.int32).view(torch.float32).item() == ref.scale_value(b)
        for n in range(1, 16):
            v = torch.tensor((n - 8) * ref.scale_value(b), dtype=torch.float64)
            assert v.to(torch.bfloat16).double() == v
        c = torch.tensor(-136 * ref.scale_value(b), dtype=torch.float64)    # the decoders' addend
        assert c.to(torch.bfloat16).double() == c


def test_handworked_row():
    """amax = 7: s = 1; halves go to the even neighbour; amax = 119 / 16 lies half-way between 17 / 16 - 1 / 16 and 17 / 16 + 1 / 16 (times 7)."""
    x = torch.zeros(64)
    x[:8] = torch.tensor([7.0, -7.0, 0.5, 1.5, -2.5, -0.5, 3.49, -6.51])
    x[32] = 119 / 16
    n, byte = ref.quantise(x)
    assert n[:8].tolist() == [15, 1, 8, 10, 6, 8, 11, 1]
    assert byte.tolist() == [20 * 8, 20 * 8]                   # 17 / 16 is the border of 1 and 9 / 8: the even byte
    data, _ = ref.pack(n, byte)
    assert data[:4].tolist() == [15 | 8 << 4, 6 | 11 << 4, 1 | 10 << 4, 8 | 1 << 4]
    assert torch.equal(ref.values(data, byte)[:8], torch.tensor([7, -7, 0, 2, -2, 0, 3, -7], dtype=torch.float64))


def test_no_value_is_off_by_more_than_half_a_step():
    x = (torch.randn(200, 128, generator=torch.Generator().manual_seed(1)) * torch.logspace(-8, 3, 200)[:, None]).bfloat16()
    _, byte = ref.quantise(x)
    step = ref.SCALES[byte].repeat_interleave(32, dim=-1)
    assert bool(((ref.held(x) - x.double()).abs() <= step / 2).all())


def test_what_is_out_of_range_saturates():
    x = torch.tensor([float("nan"), float("inf"), -float("inf"), 1e30, -30000.0, 26880.0, 1.0] + [0.0] * 25)
    assert ref.held(x)[:7].tolist() == [0.0, 26880.0, -26880.0, 26880.0, -26880.0, 26880.0, 0.0]
    assert torch.equal(ref.held(torch.zeros(32)), torch.zeros(32, dtype=torch.float64))


FAKE = 0x10000      # an aligned address that no argument check reads


def _cache_q4(**kw):
    a = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, cache_len=FAKE, n_layers=2, batch=2, n_kv_heads=2, capacity=64, head_dim=64)
    a.update(kw)
    return dlm.dlm_kv_cache_q4(*a.values())


def _cache(**kw):
    a = dict(k=FAKE, v=FAKE, cache_len=FAKE, n_layers=2, batch=2, n_kv_heads=2, capacity=64, head_dim=64)
    a.update(kw)
    return dlm.dlm_kv_cache(*a.values())


_CTX = (ctypes.c_char * 65536)()      # stands for a context: an argument error is returned before it is looked at


def _call(name, *args):
    f = getattr(ctypes.CDLL(_build.LIB), name)
    f.restype = ctypes.c_int
    conv = [ctypes.byref(a) if isinstance(a, ctypes.Structure) else ctypes.c_float(a) if isinstance(a, float) else
            ctypes.c_void_p(a) if a is None or (isinstance(a, int) and a >= FAKE) else a for a in args]
    return f(ctypes.byref(_CTX), *conv)


def commit(c, k=FAKE, v=FAKE, src_len=8, mode=0, n_max=8, lb=0, le=2):
    return _call("dlm_kv_cache_commit_q4", c, k, v, src_len, None, None, mode, None, n_max, 0, lb, le, None)


def read(c, pos=None, n_max=8, lb=0, le=2, k=FAKE, v=FAKE):
    return _call("dlm_kv_cache_read_q4", c, pos, None, n_max, lb, le, k, v, None)


def attn(c, lb=0, le=2, q=FAKE, k=FAKE, v=FAKE, heads=4, q_cap=8, out=FAKE):
    return _call("dlm_freecache_attn_step_q4", c, lb, le, q, k, v, heads, q_cap, None, 0.0, 0, out, None, FAKE, ctypes.c_size_t(1 << 40), None)


def weight(c, lb=0, le=2, q=FAKE, lse=FAKE, heads=4, q_cap=8, collected=None, decay=1.0, w=FAKE, q4=True):
    return _call("dlm_cache_weight_accumulate" + ("_q4" if q4 else ""), c, lb, le, q, lse, heads, q_cap, None, 0.0, 0, collected, decay, w, None)


def evict(c, w=FAKE, keep=32, first=0, last=0, idx=FAKE, q4=True):
    return _call("dlm_kv_cache_evict" + ("_q4" if q4 else ""), c, w, keep, first, last, idx, None, None)


def test_what_every_call_asks_of_a_4_bit_cache():
    for f in (commit, read, attn, weight, evict):
        for field in ("k", "v", "k_scale", "v_scale", "cache_len"):
            assert f(_cache_q4(**{field: None})) == dlm.DLM_ERR_NULL, (f, field)
        for field in ("n_layers", "batch", "n_kv_heads", "capacity", "head_dim"):
            for wrong in (0, -1):
                assert f(_cache_q4(**{field: wrong})) == dlm.DLM_ERR_SHAPE, (f, field)
        for wrong in (dict(head_dim=32), dict(head_dim=96), dict(head_dim=256), dict(capacity=63), dict(capacity=60), dict(k=FAKE + 8),
                      dict(v=FAKE + 4), dict(k_scale=FAKE + 8), dict(v_scale=FAKE + 2)):
            assert f(_cache_q4(**wrong)) == dlm.DLM_ERR_UNSUPPORTED, (f, wrong)


def test_refusals_of_commit_and_read():
    c = _cache_q4()
    assert commit(c, k=None) == commit(c, v=None) == read(c, k=None) == read(c, v=None) == dlm.DLM_ERR_NULL
    assert commit(c, k=FAKE + 8) == dlm.DLM_ERR_UNSUPPORTED and read(c, v=FAKE + 8) == dlm.DLM_ERR_UNSUPPORTED
    for kw in (dict(src_len=0), dict(mode=2), dict(n_max=0), dict(lb=-1), dict(le=3), dict(lb=2)):
        assert commit(c, **kw) == dlm.DLM_ERR_SHAPE, kw
    for kw in (dict(n_max=0), dict(lb=-1), dict(le=3), dict(lb=2), dict(n_max=65)):
        assert read(c, **kw) == dlm.DLM_ERR_SHAPE, kw


def test_refusals_of_attention_and_weights():
    c, cb = _cache_q4(), _cache()
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(out=None)):
        assert attn(c, **kw) == dlm.DLM_ERR_NULL, kw
    for kw in (dict(q=FAKE + 8), dict(k=FAKE + 8), dict(v=FAKE + 8), dict(out=FAKE + 8), dict(heads=3), dict(q_cap=4097)):
        assert attn(c, **kw) == dlm.DLM_ERR_UNSUPPORTED, kw
    for kw in (dict(heads=0), dict(q_cap=0), dict(lb=-1), dict(le=3), dict(lb=2)):
        assert attn(c, **kw) == dlm.DLM_ERR_SHAPE, kw
        assert weight(c, **kw) == weight(cb, q4=False, **kw) == dlm.DLM_ERR_SHAPE, kw
    for kw in (dict(q=None), dict(lse=None), dict(w=None)):
        assert weight(c, **kw) == weight(cb, q4=False, **kw) == dlm.DLM_ERR_NULL, kw
    for kw in (dict(q=FAKE + 8), dict(heads=3), dict(q_cap=4097), dict(decay=float("nan"))):
        assert weight(c, **kw) == weight(cb, q4=False, **kw) == dlm.DLM_ERR_UNSUPPORTED, kw
    assert weight(_cache(head_dim=96), q4=False) == dlm.DLM_ERR_UNSUPPORTED and weight(_cache(k=FAKE + 8), q4=False) == dlm.DLM_ERR_UNSUPPORTED
    assert weight(_cache(k=None), q4=False) == weight(_cache(cache_len=None), q4=False) == dlm.DLM_ERR_NULL
    assert attn(_cache_q4(batch=1025)) == weight(_cache_q4(batch=1025)) == dlm.DLM_ERR_UNSUPPORTED
    assert attn(_cache_q4(n_layers=1 << 20, batch=1024, capacity=1 << 20), le=1 << 20) == dlm.DLM_ERR_UNSUPPORTED     # items beyond 32 bits
    assert weight(_cache_q4(n_layers=1 << 20, batch=1024, capacity=1 << 20), le=1 << 20) == dlm.DLM_ERR_UNSUPPORTED


def test_refusals_of_eviction():
    for c, q4 in ((_cache_q4(), True), (_cache(), False)):
        assert evict(c, w=None, q4=q4) == evict(c, idx=None, q4=q4) == dlm.DLM_ERR_NULL
        for kw in (dict(keep=0), dict(keep=65), dict(keep=-3), dict(first=-1), dict(last=-1), dict(first=33), dict(first=20, last=13), dict(first=1, last=(1 << 31) - 1)):
            assert evict(c, q4=q4, **kw) == dlm.DLM_ERR_SHAPE, kw
    for kw in (dict(k=None), dict(v=None), dict(cache_len=None)):
        assert evict(_cache(**kw), q4=False) == dlm.DLM_ERR_NULL, kw
    assert evict(_cache(head_dim=12), q4=False) == evict(_cache(v=FAKE + 8), q4=False) == dlm.DLM_ERR_UNSUPPORTED
    assert evict(_cache(capacity=(1 << 20) + 1), q4=False) == dlm.DLM_ERR_UNSUPPORTED
    assert evict(_cache(n_layers=1 << 20, batch=1 << 10, capacity=1 << 10), q4=False) == dlm.DLM_ERR_UNSUPPORTED
    assert evict(_cache(batch=0), q4=False) == dlm.DLM_ERR_SHAPE


def test_workspace_size_of_wrong_arguments_is_zero():
    for c, args in ((_cache_q4(), (0, 4, 8)), (_cache_q4(), (1, 3, 8)), (_cache_q4(), (1, 4, 0)), (_cache_q4(), (1, 4, 4097)), (_cache_q4(head_dim=96), (1, 4, 8))):
        assert dlm.dlm_attn_workspace_bytes_q4(ctypes.addressof(_CTX), c, *args) == 0


def test_python_views_and_types():
    data, scale, n = torch.zeros(1, 2, 2, 8, 32, dtype=torch.uint8), torch.zeros(1, 2, 2, 8, 2, dtype=torch.uint8), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError, match="uint8"):
        dlm.make_kv_cache_q4(data.float(), data.float(), scale, scale, n)
    with pytest.raises(TypeError, match="one entry per 32"):
        dlm.make_kv_cache_q4(data, data, scale[..., :1].contiguous(), scale, n)
    with pytest.raises(TypeError, match="batch"):
        dlm.make_kv_cache_q4(data, data, scale, scale, n[:1])
    with pytest.raises(TypeError, match="CUDA"):
        dlm.make_kv_cache_q4(data, data, scale, scale, n)
    with pytest.raises(TypeError, match="expected"):      # a cache of the other kind
        dlm.dlm_kv_cache_evict_q4(None, _cache(), None, 1, 0, 0, None, None)
    with pytest.raises(TypeError, match="expected"):
        dlm.dlm_kv_cache_evict(None, _cache_q4(), None, 1, 0, 0, None, None)


def test_reference_eviction_by_hand():
    w = torch.tensor([5.0, 1.0, 4.0, 1.0, 9.0, 2.0, 2.0, float("nan")]).view(1, 1, 1, 8)
    kept, out = ref.evict(w, [7], 4, 0, 1)              # rows 4, 0, 2 and the protected 6
    assert kept[0, 0, 0].tolist() == [0, 4, 2, 6]
    assert out[0, 0, 0, :7].tolist() == [5.0, 9.0, 4.0, 2.0, 0.0, 0.0, 0.0] and bool(out[0, 0, 0, 7].isnan())
    kept, _ = ref.evict(torch.ones(1, 1, 1, 8), [8], 3, 0, 0)      # ties to the lowest rows
    assert kept[0, 0, 0].tolist() == [0, 1, 2]


def test_build_checks_the_register_counts_of_the_attention_over_4_bits():
    """Their register splits balance only at the counts that they are launched with: the build refuses any other."""
    from paper_2505_21467_b200 import build as b
    entry = "ptxas info    : Compiling entry function '_ZN3foo{}EEv' for 'sm_100a'\nptxas info    : Used {} registers\n"
    log = "".join(entry.format(part, regs) for part, regs in b.Q4_ATTENTION_REGISTERS.items())
    b.check_q4_attention_registers(log)
    for part, regs in b.Q4_ATTENTION_REGISTERS.items():
        with pytest.raises(RuntimeError):
            b.check_q4_attention_registers(log.replace(entry.format(part, regs), entry.format(part, regs - 8)))
        with pytest.raises(RuntimeError):
            b.check_q4_attention_registers(log.replace(entry.format(part, regs), ""))
