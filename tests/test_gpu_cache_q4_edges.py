"""The 4-bit cache, its attention, the rows' weights and eviction where their kernels change over: numbers of query rows and keys beside every
tile's end, scores that jump, values that are not finite, caches beyond 32-bit offsets, calls that follow each other without a pause."""
import math

import pytest
import torch

import paper_2505_21467_b200 as dlm
import q4_reference as ref
from helpers import Dev
from test_gpu_cache_evict import Plain, accumulate, check_evict, evict
from test_gpu_cache_q4 import Cache, attention_call, check_attention, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return Dev()


# query rows a KV head, by (query heads a KV head, active rows): the kernels take up to 16, 32, 128 and more
ROWS = [(1, 15), (1, 16), (1, 17), (4, 8), (3, 11), (1, 63), (2, 32), (5, 13), (1, 127), (4, 32), (3, 43), (1, 255), (8, 32), (1, 257), (7, 75)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", ROWS, ids=lambda r: f"{r[0]}x{r[1]}")
def test_numbers_of_query_rows(dev, D, rows):
    g, L = rows
    lens = [190, 64]
    lq = [L, max(1, L - 3)]
    c = Cache(dev, 1, 2, 2, 192, D, lens, 200 + L)
    q, kn, vn = inputs(1, 2, 2 * g, 2, L, D, lq, 201)
    out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), torch.tensor(lq, dtype=torch.int32, device="cuda"))
    assert dev.status() == 0
    check_attention(c, q, kn, vn, lq, out, lse)
    weight = dev.guarded((1, 2, 2, 192), torch.float32, -1.0)
    accumulate(dev, c, q.cuda(), lse, torch.tensor(lq, dtype=torch.int32, device="cuda"), None, 0.0, weight)
    assert dev.status() == 0
    want, most = ref.weights(c.values("k", 0), lens, q[0], lse[0].cpu(), lq, None, 0.0)
    seen = ~want.isnan()
    rel = 2 * D * 2.0 ** -24 * most + 2.0 ** -22 * most + 2.0 ** -20 + g * L * 2.0 ** -24
    assert bool(((weight[0].cpu().double() - want).abs() <= rel * want + 2.0 ** -120)[seen].all())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g,L", [(1, 1), (2, 12), (1, 40), (7, 20)])
def test_numbers_of_keys(dev, D, g, L):
    for cached in (0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 191, 193, 255, 256, 257, 320, 383):
        c = Cache(dev, 1, 1, 1, (cached + 8) // 8 * 8, D, [cached], cached)
        q, kn, vn = inputs(1, 1, g, 1, L, D, [L], 211)
        out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None)
        assert dev.status() == 0, cached
        check_attention(c, q, kn, vn, [L], out, lse)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g,L", [(1, 3), (2, 15), (4, 20), (6, 40)])
@pytest.mark.parametrize("where", [[70], [130, 131, 400], [3, 200, 1000, 1300], [1399]])
def test_scores_that_jump(dev, D, g, L, where):
    """Rows whose scores are far above all before (hundreds of units: beyond any reference that the first keys give), each further than the
    last; the other rows then have no weight, and the sums begin anew."""
    C = 1400
    c = Cache(dev, 1, 1, 1, C, D, [C], 221)
    k = torch.randn(1, 1, 1, C, D, generator=torch.Generator().manual_seed(222)) * 0.01
    for i, row in enumerate(where):
        k[..., row, :] = 40.0 * (i + 1)
    c.host["k"], c.host["k_scale"] = ref.pack(*ref.quantise(k.bfloat16()))
    c.gpu["k"].copy_(c.host["k"]), c.gpu["k_scale"].copy_(c.host["k_scale"])
    q, kn, vn = inputs(1, 1, g, 1, L, D, [L], 223)
    q = q.abs()
    q[..., 0::2] = 0.5
    kn = (kn.float() * 0.01).bfloat16()
    out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None)
    assert dev.status() == 0
    check_attention(c, q, kn, vn, [L], out, lse)
    # and the same the other way round: the first key has nearly all
    kn[..., 0, :] = 300.0
    out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None)
    assert dev.status() == 0
    check_attention(c, q, kn, vn, [L], out, lse)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g,L", [(1, 2), (2, 14), (2, 30), (7, 24)])
def test_what_is_not_finite_stays_with_its_rows(dev, D, g, L):
    """A NaN or an infinity in a fresh key or a query reaches the rows whose formula has it, and no others."""
    B, lens = 3, [150, 70, 0]
    c = Cache(dev, 1, B, 2, 152, D, lens, 231)
    q, kn, vn = inputs(1, B, 2 * g, 2, L, D, [L] * B, 232)
    kn[0, 0, 1, L - 1, 3] = float("nan")          # sequence 0, KV head 1: every row
    q[0, 1, 0, 0, 5] = float("nan")               # sequence 1, query head 0, row 0
    vn[0, 2, 0, 0, 7] = float("inf")              # sequence 2, KV head 0: column 7 of every row
    out, lse = (t.cpu() for t in attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None))
    assert dev.status() == 0
    assert bool(out[0, 0, g:].isnan().all()) and bool(lse[0, 0, g:].isnan().all())
    assert bool(out[0, 1, 0, 0].isnan().all()) and bool(lse[0, 1, 0, 0].isnan())
    assert bool((out[0, 2, :g, :, 7] == float("inf")).all())
    kn2, q2, vn2 = kn.clone(), q.clone(), vn.clone()
    kn2[0, 0, 1, L - 1, 3] = q2[0, 1, 0, 0, 5] = vn2[0, 2, 0, 0, 7] = 0.0
    clean = torch.ones_like(out, dtype=torch.bool)
    clean[0, 0, g:] = clean[0, 1, 0, 0] = clean[0, 2, :g, :, 7] = False
    want, w_lse, spread, size = ref.attention(c.values("k", 0), c.values("v", 0), lens, q2[0], kn2[0], vn2[0], [L] * B)
    off = size * 2 * D * 2.0 ** -24 + 2.0 ** -20
    tol = 2.0 ** -8 * (spread + want.abs()) * (1 + 2.0 ** -6) + 2 * off[..., None] * spread
    assert bool(((out[0].double() - want).abs() <= tol)[clean[0]].all())


def test_weights_with_logarithms_that_are_not_finite(dev):
    D, L, C = 128, 9, 140
    c = Plain(dev, 1, 1, 1, 144, D, [C], 241)
    q, kn, vn = inputs(1, 1, 2, 1, L, D, [L], 242)
    _, lse, _, _ = ref.attention(c.values("k", 0), c.values("v", 0), [C], q[0], kn[0], vn[0], [L])
    lse = lse.float()[None]
    lse[0, 0, 0, 1], lse[0, 0, 1, 2] = -math.inf, math.inf        # left out; no weight
    weight = dev.guarded((1, 1, 1, 144), torch.float32, 0.0)
    accumulate(dev, c, q.cuda(), lse.cuda(), None, None, 1.0, weight)
    assert dev.status() == 0
    keep = lse.clone()
    keep[0, 0, 1, 2] = -math.inf
    want, most = ref.weights(c.values("k", 0), [C], q[0], keep[0], [L], None, 1.0)
    rel = 2 * D * 2.0 ** -24 * most + 2.0 ** -22 * most + 2.0 ** -20 + 2 * L * 2.0 ** -24
    assert bool(((weight[0, 0, 0, :C].cpu().double() - want[0, 0, :C]).abs() <= rel * want[0, 0, :C]).all())
    lse[0, 0, 0, 0] = math.nan
    accumulate(dev, c, q.cuda(), lse.cuda(), None, None, 1.0, weight)
    assert dev.status() == 0
    assert bool(weight[0, 0, 0, :C].isnan().all()) and bool((weight[0, 0, 0, C:] == 0).all())


def test_offsets_beyond_32_bits(dev):
    """Caches of more than 2^32 bytes and rows beyond 2^31 values: the last head of the last layer."""
    NL, B, H, D, capacity = 17, 2, 2, 128, 1 << 20                   # 4.6 GB of K and of V; every row but the last head's first ones unseen
    k, v = (torch.zeros(NL, B, H, capacity, D // 2, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(NL, B, H, capacity, D // 32, dtype=torch.uint8, device="cuda") for _ in range(2))
    assert k.numel() > 1 << 32
    n = torch.tensor([0, 300], dtype=torch.int32, device="cuda")
    view = dlm.make_kv_cache_q4(k, v, ks, vs, n)
    g = torch.Generator().manual_seed(251)
    kn, vn = (torch.randn(1, B, H, 300, D, generator=g).bfloat16() for _ in range(2))
    n.zero_()
    dlm.dlm_kv_cache_commit_q4(dev.ctx, view, kn.cuda(), vn.cuda(), 300, None, None, dlm.DLM_DST_APPEND, torch.tensor([0, 300], dtype=torch.int32, device="cuda"), 300, 1,
                               NL - 1, NL)
    ko, vo = (torch.zeros(1, B, H, 300, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dlm.dlm_kv_cache_read_q4(dev.ctx, view, None, None, 300, NL - 1, NL, ko, vo)
    assert dev.status() == 0
    assert torch.equal(ko[:, 1].cpu().double(), ref.held(kn[:, 1])) and torch.equal(vo[:, 1].cpu().double(), ref.held(vn[:, 1]))
    q, k2, v2 = inputs(1, B, 4, H, 3, D, [3, 3], 252)
    out, lse = torch.empty_like(q, device="cuda"), torch.empty(1, B, 4, 3, device="cuda")
    ws = dev.workspace(dlm.dlm_attn_workspace_bytes_q4(dev.ctx, view, 1, 4, 3))
    dlm.dlm_freecache_attn_step_q4(dev.ctx, view, NL - 1, NL, q.cuda(), k2.cuda(), v2.cuda(), 4, 3, None, 0.0, 300, out, lse, ws)
    weight = torch.zeros(NL, B, H, capacity, device="cuda")
    dlm.dlm_cache_weight_accumulate_q4(dev.ctx, view, NL - 1, NL, q.cuda(), lse, 4, 3, None, 0.0, 300, None, 1.0, weight)
    assert dev.status() == 0
    full = torch.zeros(B, H, 300, D, dtype=torch.float64), torch.zeros(B, H, 300, D, dtype=torch.float64)
    for t, new in zip(full, (kn, vn)):
        t[1] = ref.held(new[0, 1])
    want, w_lse, spread, _ = ref.attention(full[0], full[1], [0, 300], q[0], k2[0], v2[0], [3, 3])
    assert bool(((out[0].cpu().double() - want).abs() <= 2.0 ** -7 * (spread + want.abs())).all())
    w, _ = ref.weights(full[0], [0, 300], q[0], lse[0].cpu(), [3, 3], None, 1.0)
    assert torch.allclose(weight[NL - 1, 1, :, :300].cpu().double(), w[1], rtol=1e-4)
    assert bool((weight[NL - 1, 1, :, 300:] == 0).all()) and bool((weight[:NL - 1] == 0).all())


def test_eviction_beyond_32_bits_and_of_a_million_rows(dev):
    NL, B, H, D, capacity = 3, 1, 3, 128, 1 << 20                   # 2.4 GB each, above 2^31 bytes
    k, v = (torch.empty(NL, B, H, capacity, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows = torch.arange(capacity, device="cuda", dtype=torch.float32)
    k[..., 0], k[..., 1] = (rows % 256).bfloat16(), (rows // 256 % 256).bfloat16()
    k[..., 2] = (rows // 65536).bfloat16()
    v.copy_(k)
    length, keep = capacity - 5, 700001
    n = torch.tensor([length], dtype=torch.int32, device="cuda")
    weight = torch.rand(NL, B, H, capacity, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    weight = (weight * 1000).floor()                                # many ties
    kept = torch.empty(NL, B, H, keep, dtype=torch.int32, device="cuda")
    dlm.dlm_kv_cache_evict(dev.ctx, dlm.make_kv_cache(k, v, n), weight, keep, 3, 4, kept, None)
    assert dev.status() == 0 and n.tolist() == [keep]
    for l, h in ((0, 0), (NL - 1, H - 1)):
        w = weight[l, 0, h, :length].clone()
        w[:3] = w[length - 4:] = math.inf
        stay = torch.zeros(length, dtype=torch.bool, device="cuda")
        stay[w.argsort(descending=True, stable=True)[:keep]] = True
        idx = torch.arange(keep, device="cuda")
        idx[~stay[:keep]] = torch.nonzero(stay[keep:]).flatten() + keep
        assert torch.equal(kept[l, 0, h].long(), idx)
        for t in (k, v):
            assert torch.equal((t[l, 0, h, :keep, 0].double() + 256 * t[l, 0, h, :keep, 1].double() + 65536 * t[l, 0, h, :keep, 2].double()).long(), idx)


@pytest.mark.parametrize("kind", [Cache, Plain])
def test_calls_right_behind_each_other(dev, kind):
    """A loop of every call, once with a pause after each and once without: the same bits."""
    NL, B, Hq, H, D, L, capacity, keep = 3, 2, 8, 2, 128, 16, 160, 100
    q4 = kind is Cache
    attn = dlm.dlm_freecache_attn_step_q4 if q4 else dlm.dlm_freecache_attn_step
    bytes_of = dlm.dlm_attn_workspace_bytes_q4 if q4 else dlm.dlm_attn_workspace_bytes
    collect = dlm.dlm_cache_weight_accumulate_q4 if q4 else dlm.dlm_cache_weight_accumulate
    commit = dlm.dlm_kv_cache_commit_q4 if q4 else dlm.dlm_kv_cache_commit
    throw_out = dlm.dlm_kv_cache_evict_q4 if q4 else dlm.dlm_kv_cache_evict
    steps = [[t.cuda() for t in inputs(NL, B, Hq, H, L, D, [L, L], 260 + i)] for i in range(8)]
    results = []
    for pause in (True, False):
        c = kind(dev, NL, B, H, capacity, D, [90, 30], 261)
        ws = torch.empty(bytes_of(dev.ctx, c.view, NL, Hq, L) + 256, dtype=torch.uint8, device="cuda")
        weight, kept = torch.zeros(NL, B, H, capacity, device="cuda"), torch.empty(NL, B, H, keep, dtype=torch.int32, device="cuda")
        outs = []
        torch.cuda.synchronize()
        for q, kn, vn in steps:
            out, lse = torch.empty_like(q), torch.empty(NL, B, Hq, L, device="cuda")
            for call in (lambda: attn(dev.ctx, c.view, 0, NL, q, kn, vn, Hq, L, None, 0.0, 0, out, lse, ws),
                         lambda: collect(dev.ctx, c.view, 0, NL, q, lse, Hq, L, None, 0.0, 0, weight, 0.9, weight),
                         lambda: commit(dev.ctx, c.view, kn, vn, L, None, None, dlm.DLM_DST_APPEND, None, L, 1, 0, NL),
                         lambda: throw_out(dev.ctx, c.view, weight, keep, 2, L, kept, weight)):
                call()
                if pause:
                    torch.cuda.synchronize()
            outs += [out, lse]
        outs += [weight, kept, c.cache_len, *c.gpu.values()]
        assert dev.status() == 0
        results.append([t.clone() for t in outs])
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert results[0][-1 - len(c.gpu)].tolist() == [100, 100]


def test_a_batch_of_many_sequences_with_gaps(dev):
    """Sequences of all lengths, empty and inactive ones among them, in every kernel's order of units."""
    B, H, D, L = 37, 1, 64, 6
    lens = [(37 * b * b) % 211 if b % 5 else 0 for b in range(B)]
    lq = [0 if b % 7 == 3 else 1 + b % L for b in range(B)]
    c = Cache(dev, 2, B, H, 216, D, lens, 271)
    q, kn, vn = inputs(2, B, 2, H, L, D, lq, 272)
    q_len = torch.tensor(lq, dtype=torch.int32, device="cuda")
    out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), q_len)
    assert dev.status() == 0
    check_attention(c, q, kn, vn, lq, out, lse)
    weight = dev.guarded((2, B, H, 216), torch.float32, 4.0)
    accumulate(dev, c, q.cuda(), lse, q_len, weight, 1.0, weight)
    for l in range(2):
        want, most = ref.weights(c.values("k", l), lens, q[l], lse[l].cpu(), lq, torch.full((B, H, 216), 4.0), 1.0)
        seen = ~want.isnan()
        assert torch.allclose(weight[l].cpu().double()[seen], want[seen], rtol=2 * D * 2.0 ** -24 * most + 2.0 ** -19, atol=2.0 ** -21)
    check_evict(dev, c, weight.cpu().clone(), lens, 100, 1, 1)


def test_hints_of_any_size_give_the_same_results(dev):
    c = Cache(dev, 2, 2, 2, 1024, 128, [1000, 20], 281)
    q, kn, vn = inputs(2, 2, 4, 2, 10, 128, [10, 10], 282)
    ws = torch.empty(dlm.dlm_attn_workspace_bytes_q4(dev.ctx, c.view, 2, 4, 10), dtype=torch.uint8, device="cuda")
    for hint in (-5, 0, 1, 64, 1024, 1 << 30):
        out, lse = torch.empty_like(q, device="cuda"), torch.empty(2, 2, 4, 10, device="cuda")
        dlm.dlm_freecache_attn_step_q4(dev.ctx, c.view, 0, 2, q.cuda(), kn.cuda(), vn.cuda(), 4, 10, None, 0.0, hint, out, lse, ws)
        weight = torch.zeros(2, 2, 2, 1024, device="cuda")
        dlm.dlm_cache_weight_accumulate_q4(dev.ctx, c.view, 0, 2, q.cuda(), lse, 4, 10, None, 0.0, hint, None, 1.0, weight)
        assert dev.status() == 0
        check_attention(c, q, kn, vn, [10, 10], out, lse)
        w, _ = ref.weights(c.values("k", 1), [1000, 20], q[1], lse[1].cpu(), [10, 10], None, 1.0)
        assert torch.allclose(weight[1, 0, :, :1000].cpu().double(), w[0, :, :1000], rtol=1e-4)


@pytest.mark.parametrize("low", [-math.inf, -3e38, -1e30, -3e4])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g,L", [(1, 3), (2, 15), (4, 20), (6, 40)])
def test_fresh_keys_far_below_the_others(dev, g, L, D, low):
    """Fresh rows whose scores are the lowest numbers or -infinity for every query have no weight, wherever they are: as the first key, as the only ones
    of a tile or of a block's part.  The others' weights are as if those rows were not there (differences of thousands of units are 0 in 64 bits too)."""
    for cached in (0, 5, 64, 130, 3000):
        c = Cache(dev, 1, 1, 1, (cached + 8) // 8 * 8, D, [cached], 291)
        q, kn, vn = inputs(1, 1, g, 1, L, D, [L], 292)
        q[..., 0] = q[..., 0].abs() + 1
        for rows in (slice(0, 1), slice(0, L - 1), slice(0, L)):
            if rows.stop == L and cached == 0:
                continue
            low_kn = kn.clone()
            low_kn[..., rows, 0] = low
            out, lse = (t.cpu() for t in attention_call(dev, c, q.cuda(), low_kn.cuda(), vn.cuda(), None))
            assert dev.status() == 0
            want, w_lse, spread, size = ref.attention(c.values("k", 0), c.values("v", 0), [cached], q[0], kn[0, :, :, rows.stop:], vn[0, :, :, rows.stop:], [L])
            off = size * 2 * D * 2.0 ** -24 + 2.0 ** -20              # as check_attention has it
            tol = 2.0 ** -8 * (spread + want.abs()) * (1 + 2.0 ** -6) + 2 * off[..., None] * spread + 2.0 ** -110
            assert bool(((out[0].double() - want).abs() <= tol).all()), (cached, rows)
            assert bool(((lse[0].double() - w_lse).abs() <= off + 2.0 ** -22 * (w_lse.abs() + 8)).all()), (cached, rows)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("g,L", [(1, 3), (2, 15), (4, 20), (6, 40)])
def test_a_first_key_far_below_and_scores_that_differ_among_the_others(dev, g, L, D):
    """The first key's score is no scale for the others': theirs differ by tens of units and keep their differences."""
    cached = 700
    c = Cache(dev, 1, 1, 1, 704, D, [cached], 301)
    k = torch.randn(1, 1, 1, 704, D, generator=torch.Generator().manual_seed(302)) * 4
    k[..., 0, :] = 0
    k[..., 0, :32] = -26000.0
    k[..., 128, :32] = -20000.0
    c.host["k"], c.host["k_scale"] = ref.pack(*ref.quantise(k.bfloat16()))
    c.gpu["k"].copy_(c.host["k"]), c.gpu["k_scale"].copy_(c.host["k_scale"])
    q, kn, vn = inputs(1, 1, g, 1, L, D, [L], 303)
    q[..., :32] = q[..., :32].abs() + 0.5
    out, lse = (t.cpu() for t in attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None))
    assert dev.status() == 0
    seen = torch.ones(cached, dtype=torch.bool)
    seen[0] = seen[128] = False                                     # scores below -10^4: no weight
    want, w_lse, spread, size = ref.attention(c.values("k", 0)[:, :, :cached][:, :, seen], c.values("v", 0)[:, :, :cached][:, :, seen], [cached - 2], q[0], kn[0], vn[0], [L])
    off = size * 2 * D * 2.0 ** -24 + 2.0 ** -20
    tol = 2.0 ** -8 * (spread + want.abs()) * (1 + 2.0 ** -6) + 2 * off[..., None] * spread + 2.0 ** -110
    assert bool(((out[0].double() - want).abs() <= tol).all())
    assert bool(((lse[0].double() - w_lse).abs() <= off + 2.0 ** -22 * (w_lse.abs() + 8)).all())


def test_nothing_collected_takes_no_decay(dev):
    c = Cache(dev, 1, 1, 1, 64, 64, [40], 311)
    q, kn, vn = inputs(1, 1, 2, 1, 3, 64, [3], 312)
    _, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None)
    one, two = (dev.guarded((1, 1, 1, 64), torch.float32, 0.0) for _ in range(2))
    accumulate(dev, c, q.cuda(), lse, None, None, 0.5, one)
    accumulate(dev, c, q.cuda(), lse, None, None, math.inf, two)
    assert dev.status() == 0 and torch.equal(one, two) and bool((one[..., :40] > 0).all())


@pytest.mark.parametrize("D,g,L", [(128, 17, 1), (128, 1, 2), (128, 3, 12), (128, 1, 130), (64, 32, 1)])
def test_the_largest_batch(dev, D, g, L):
    """1024 sequences, whose lengths take what shared memory a kernel has left."""
    B = 1024
    lens, lq = [(7 * b) % 24 for b in range(B)], [(b % (L + 1)) if b % 3 else L for b in range(B)]
    c = Cache(dev, 1, B, 1, 24, D, lens, 321)
    q, kn, vn = inputs(1, B, g, 1, L, D, lq, 322)
    q_len = torch.tensor(lq, dtype=torch.int32, device="cuda")
    out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), q_len)
    assert dev.status() == 0
    check_attention(c, q, kn, vn, lq, out, lse)
    weight = dev.guarded((1, B, 1, 24), torch.float32, 0.0)
    accumulate(dev, c, q.cuda(), lse, q_len, None, 0.0, weight)
    assert dev.status() == 0
    want, most = ref.weights(c.values("k", 0), lens, q[0], lse[0].cpu(), lq, None, 0.0)
    seen = ~want.isnan()
    rel = 2 * D * 2.0 ** -24 * most + 2.0 ** -22 * most + 2.0 ** -20 + g * L * 2.0 ** -24
    assert bool(((weight[0].cpu().double() - want).abs() <= rel * want + 2.0 ** -120)[seen].all())


def test_a_length_out_of_range_in_the_largest_batch(dev):
    """... is clamped and reported there too."""
    B, D = 1024, 128
    c = Cache(dev, 1, B, 1, 24, D, [10] * B, 331)
    q, kn, vn = inputs(1, B, 20, 1, 1, D, [1] * B, 332)
    out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None)
    assert dev.status() == 0
    for wrong, same in ((1 << 30, 24), (-3, 0)):
        c.cache_len[500] = same
        want, w_lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None)
        assert dev.status() == 0
        c.cache_len[500] = wrong
        got, g_lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None)
        assert dev.status() == dlm.DLM_ERR_CAPACITY
        assert torch.equal(got, want) and torch.equal(g_lse, w_lse)
