"""Attention weights of cached rows against the 64-bit form; eviction bit for bit; and both with attention and commit, as they are used."""
import pytest
import torch

import paper_2505_21467_b200 as dlm
import q4_reference as ref
from helpers import Dev, gpu_attn_step
from test_gpu_cache_q4 import Cache, attention_call, check_attention, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return Dev()


class Plain:
    """A bf16 cache with the same interface; rows that nobody sees are NaN."""

    def __init__(self, dev, NL, B, H, capacity, D, lens, seed):
        g = torch.Generator().manual_seed(seed)
        self.shape = (NL, B, H, capacity, D)
        self.host = {"k": torch.randn(NL, B, H, capacity, D, generator=g), "v": torch.randn(NL, B, H, capacity, D, generator=g)}
        self.host["k"][..., 5::16] *= 8
        for b, n in enumerate(lens):
            for t in self.host.values():
                t[:, b, :, n:] = float("nan")
        self.host = {n: t.bfloat16() for n, t in self.host.items()}
        self.gpu = {n: dev.guarded(tuple(t.shape), torch.bfloat16, 0) for n, t in self.host.items()}
        for n, t in self.host.items():
            self.gpu[n].copy_(t)
        self.cache_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.view = dlm.make_kv_cache(self.gpu["k"], self.gpu["v"], self.cache_len)

    def values(self, n, layer):
        return self.host[n][layer]


def accumulate(dev, c, q, lse, q_len, collected, decay, weight, layers=None, scale=0.0):
    lb, le = layers or (0, c.shape[0])
    call = dlm.dlm_cache_weight_accumulate_q4 if isinstance(c, Cache) else dlm.dlm_cache_weight_accumulate
    call(dev.ctx, c.view, lb, le, q, lse, q.shape[2], q.shape[3], q_len, scale, 0, collected, decay, weight)


WEIGHT_CASES = [
    # NL, B, Hq, H, D, L, cached rows, active rows
    (1, 1, 1, 1, 64, 1, [1], [1]),
    (1, 1, 4, 2, 64, 32, [256], [32]),
    (1, 1, 28, 4, 128, 32, [1024], [32]),
    (2, 3, 8, 2, 128, 5, [63, 0, 129], [5, 3, 0]),                  # an empty cache; a sequence without active rows
    (3, 2, 4, 4, 128, 1, [200, 777], [1, 1]),
    (1, 2, 8, 2, 128, 77, [100, 300], [77, 64]),                    # more query rows than two slots: they go through
    (2, 1, 8, 1, 64, 100, [1300], [100]),
    (40, 2, 4, 4, 64, 4, [90, 257], [4, 2]),
    (1, 1, 8, 2, 64, 33, [9000], [33]),
]


@pytest.mark.parametrize("kind", [Cache, Plain])
@pytest.mark.parametrize("case", WEIGHT_CASES, ids=lambda c: "-".join(map(str, c[:6])))
def test_weights_match_64_bits(dev, kind, case):
    """Tolerance, relative: a score is off by at most 2 D roundings of sum |q k| scale, its exponent by three more of |score| + |lse|, the
    exponential by 2^-21 and the sum by a rounding a term; absolute: a rounding of what was collected."""
    NL, B, Hq, H, D, L, lens, lq = case
    capacity = (max(lens) + 15) // 8 * 8
    c = kind(dev, NL, B, H, capacity, D, lens, 121)
    q, kn, vn = inputs(NL, B, Hq, H, L, D, lq, 122)
    lse = torch.stack([ref.attention(c.values("k", l), c.values("v", l), lens, q[l], kn[l], vn[l], lq)[1] for l in range(NL)]).float()
    collected = torch.rand(NL, B, H, capacity, generator=torch.Generator().manual_seed(3))
    q_len = None if lq == [L] * B else torch.tensor(lq, dtype=torch.int32, device="cuda")
    for given, decay, in_place in ((None, 1.0, False), (collected, 0.5, False), (collected, 1.0, True), (torch.full_like(collected, float("nan")), 0.0, False)):
        weight = dev.guarded((NL, B, H, capacity), torch.float32, -5.0)
        src = None if given is None else given.cuda()
        if in_place:
            weight.copy_(given)
            src = weight
        accumulate(dev, c, q.cuda(), lse.cuda(), q_len, src, decay, weight)
        got = weight.cpu().double()
        assert dev.status() == 0
        for l in range(NL):
            want, most = ref.weights(c.values("k", l), lens, q[l], lse[l], lq, None if given is None else given[l], decay)
            seen = ~want.isnan()
            rel = 2 * D * 2.0 ** -24 * most + 2.0 ** -22 * most + 2.0 ** -20 + (Hq // H) * L * 2.0 ** -24
            assert bool(((got[l] - want).abs() <= rel * want.abs() + 2.0 ** -23)[seen].all()), float(((got[l] - want).abs() / want.abs())[seen].max())
            untouched = given[l].double() if in_place else torch.full_like(got[l], -5.0)
            assert torch.equal(got[l][~seen], untouched[~seen])


def test_weights_of_a_layer_range_leave_the_others(dev):
    c = Cache(dev, 4, 1, 2, 64, 64, [50], 131)
    q, kn, vn = inputs(2, 1, 4, 2, 3, 64, [3], 132)
    lse = torch.zeros(2, 1, 4, 3)
    lse[0, 0, 1, 1] = -float("inf")                                # a row that is left out
    weight = dev.guarded((4, 1, 2, 64), torch.float32, 2.0)
    accumulate(dev, c, q.cuda(), lse.cuda(), None, weight, 0.25, weight, layers=(1, 3), scale=0.02)
    assert dev.status() == 0
    for l in (0, 3):
        assert bool((weight[l] == 2.0).all())
    for l in (1, 2):
        want, most = ref.weights(c.values("k", l), [50], q[l - 1], lse[l - 1], [3], torch.full((1, 2, 64), 2.0), 0.25, scale=0.02)
        assert torch.allclose(weight[l, 0, :, :50].cpu().double(), want[0, :, :50], rtol=2 * 64 * 2.0 ** -24 * most + 2.0 ** -19, atol=0)


def evict(dev, c, weight, keep, first=0, last=0, out=None):
    kept = dev.guarded(tuple(weight.shape[:3]) + (keep,), torch.int32, -7)
    call = dlm.dlm_kv_cache_evict_q4 if isinstance(c, Cache) else dlm.dlm_kv_cache_evict
    call(dev.ctx, c.view, weight, keep, first, last, kept, out)
    return kept


def check_evict(dev, c, weight, lens, keep, first, last, in_place=False):
    before = {n: t.clone() for n, t in c.gpu.items()}
    w = dev.guarded(tuple(weight.shape), torch.float32, 0.0)
    w.copy_(weight)
    out = w if in_place else dev.guarded(tuple(weight.shape), torch.float32, -3.0)
    kept = evict(dev, c, w, keep, first, last, out)
    assert dev.status() == 0
    want, want_w = ref.evict(weight, lens, keep, first, last)
    assert torch.equal(kept.cpu(), want)
    left = weight if in_place else torch.full_like(weight, -3.0)
    want_w = torch.where(torch.zeros_like(weight, dtype=torch.bool), want_w, want_w)
    for b, n in enumerate(lens):
        assert torch.equal(out[:, b, :, n:].cpu().nan_to_num(7.5), left[:, b, :, n:].nan_to_num(7.5))
        assert torch.equal(out[:, b, :, :n].cpu().nan_to_num(7.5), want_w[:, b, :, :n].nan_to_num(7.5))
    for name, t in before.items():                                 # moved rows in their places, every other row as it was
        at = torch.arange(t.shape[3], device="cuda").expand(t.shape[:4]).clone()
        at[..., :keep] = torch.where(kept >= 0, kept, at[..., :keep])
        moved = t.gather(3, at[..., None].expand(t.shape))
        assert torch.equal(moved.view(torch.uint8), c.gpu[name].contiguous().view(torch.uint8)), name
    assert c.cache_len.tolist() == [min(n, keep) for n in lens]


EVICT_CASES = [
    # NL, B, H, D, lengths, keep, first, last
    (1, 1, 1, 64, [1], 1, 0, 0),
    (1, 1, 1, 64, [2], 1, 0, 1),
    (2, 3, 2, 128, [45, 0, 7], 20, 2, 5),                           # nothing cached; fewer rows than are kept
    (1, 2, 4, 128, [300, 299], 299, 0, 0),
    (3, 2, 2, 64, [1000, 777], 1, 0, 0),
    (28, 2, 4, 128, [1152, 900], 700, 0, 64),
    (1, 1, 2, 64, [4096], 2048, 16, 16),                            # the last length of one tile of the short kernel, and the next
    (1, 1, 2, 64, [4097], 2048, 0, 0),
    (1, 2, 1, 64, [16384, 16000], 5000, 1, 1),
    (1, 2, 1, 64, [16385, 40000], 20000, 100, 100),                 # several tiles
    (1, 1, 1, 64, [50001], 49999, 0, 0),
    (1, 1, 1, 64, [33000], 100, 0, 0),
]


@pytest.mark.parametrize("kind", [Cache, Plain])
@pytest.mark.parametrize("case", EVICT_CASES, ids=lambda c: "-".join(map(str, (*c[:4], max(c[4]), c[5]))))
def test_evict_keeps_what_the_definition_keeps(dev, kind, case):
    NL, B, H, D, lens, keep, first, last = case
    capacity = (max(lens) + 15) // 8 * 8
    g = torch.Generator().manual_seed(141)
    weight = torch.rand(NL, B, H, capacity, generator=g).reciprocal().sqrt()
    c = kind(dev, NL, B, H, capacity, D, lens, 142)
    check_evict(dev, c, weight, lens, keep, first, last)
    c.cache_len.copy_(torch.tensor(lens))
    few = torch.randint(-2, 3, weight.shape, generator=g).float() * 0.5          # ties everywhere, -0 and 0 among them
    few[torch.rand(weight.shape, generator=g) < 0.05] = -0.0
    few[torch.rand(weight.shape, generator=g) < 0.03] = float("nan")
    few[torch.rand(weight.shape, generator=g) < 0.03] = float("inf")
    few[torch.rand(weight.shape, generator=g) < 0.03] = -float("inf")
    check_evict(dev, c, few, lens, keep, first, last, in_place=True)


@pytest.mark.parametrize("kind", [Cache, Plain])
def test_weights_in_order_and_all_alike(dev, kind):
    for weight in (torch.arange(640.0), -torch.arange(640.0), torch.zeros(640), torch.full((640,), float("nan")), torch.full((640,), 1e-42)):
        c = kind(dev, 1, 1, 1, 640, 64, [633], 151)
        check_evict(dev, c, weight.expand(1, 1, 1, 640).contiguous(), [633], 300, 0, 0)


def test_a_head_size_that_only_the_commit_takes(dev):
    lens, g = [50, 33], torch.Generator().manual_seed(5)
    c = Plain(dev, 2, 2, 3, 56, 24, lens, 152)
    check_evict(dev, c, torch.rand(2, 2, 3, 56, generator=g), lens, 20, 0, 0)


def test_a_length_out_of_range_evicts_nothing(dev):
    c = Cache(dev, 1, 2, 2, 64, 64, [64, 60], 161)
    before = {n: t.clone() for n, t in c.gpu.items()}
    c.cache_len.copy_(torch.tensor([65, -1]))
    out = dev.guarded((1, 2, 2, 64), torch.float32, 1.0)
    kept = evict(dev, c, torch.rand(1, 2, 2, 64, device="cuda"), 30, out=out)
    assert dev.status() == dlm.DLM_ERR_CAPACITY
    assert c.cache_len.tolist() == [65, -1] and bool((kept == -1).all()) and bool((out == 1.0).all())
    assert all(torch.equal(before[n], c.gpu[n]) for n in before)


@pytest.mark.parametrize("kind", [Cache, Plain])
def test_a_serving_loop_with_eviction(dev, kind):
    """Windows of a block are attended to, their rows' attention collected, the block committed, and every time the cache is over its limit
    it is brought down; what is in it at every step is followed on the host, row by row."""
    NL, B, Hq, H, D, L, keep, capacity = 2, 2, 4, 2, 64, 24, 60, 112
    c = kind(dev, NL, B, H, capacity, D, [0, 0], 171)
    weight = torch.zeros(NL, B, H, capacity, device="cuda")
    length = 0
    for step in range(6):
        q, kn, vn = inputs(NL, B, Hq, H, L, D, [L, L], 172 + step)
        if kind is Cache:
            out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None)
            commit = dlm.dlm_kv_cache_commit_q4
            now = {n: torch.stack([c.values(n, l) for l in range(NL)]) for n in ("k", "v")}
        else:
            out, lse = gpu_attn_step(dev, c.gpu["k"], c.gpu["v"], c.cache_len, q.cuda(), kn.cuda(), vn.cuda())
            commit = dlm.dlm_kv_cache_commit
            now = c.host
        before = weight.cpu()
        accumulate(dev, c, q.cuda(), lse, None, weight, 0.9, weight)
        assert dev.status() == 0
        check_attention(c, q, kn, vn, [L, L], out, lse)
        for l in range(NL):
            want, most = ref.weights(now["k"][l], [length] * B, q[l], lse[l].cpu(), [L, L], before[l], 0.9)
            seen = ~want.isnan()
            assert torch.allclose(weight[l].cpu().double()[seen], want[seen], rtol=2 * D * 2.0 ** -24 * most + 2.0 ** -19 + L * Hq * 2.0 ** -24, atol=2.0 ** -23)
        commit(dev.ctx, c.view, kn.cuda(), vn.cuda(), L, None, None, dlm.DLM_DST_APPEND, None, L, 1, 0, NL)
        length += L
        c.host = {n: t.cpu() for n, t in c.gpu.items()}
        if length > keep + L:
            w = weight.cpu()
            check_evict(dev, c, w, [length] * B, keep, 4, L)
            weight.copy_(w)
            weight_out = weight                                     # and the weights with the rows
            c.cache_len.fill_(length)
            for n in c.gpu:
                c.gpu[n].copy_(c.host[n])
            evict(dev, c, weight, keep, 4, L, weight_out)
            assert dev.status() == 0
            length = keep
            c.host = {n: t.cpu() for n, t in c.gpu.items()}
        assert c.cache_len.tolist() == [length] * B
    assert length == keep + L or length == keep


def test_eviction_in_a_graph_and_on_another_stream(dev):
    lens, keep = [300, 200], 128
    c = Plain(dev, 2, 2, 2, 304, 64, lens, 181)
    g = torch.Generator().manual_seed(4)
    weight = torch.rand(2, 2, 2, 304, generator=g).cuda()
    kept, out = torch.zeros(2, 2, 2, keep, dtype=torch.int32, device="cuda"), torch.zeros_like(weight)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        dlm.dlm_kv_cache_evict(dev.ctx, c.view, weight, keep, 0, 0, kept, out)
    for seed in range(3):
        w = torch.rand(2, 2, 2, 304, generator=torch.Generator().manual_seed(seed))
        weight.copy_(w)
        c.cache_len.copy_(torch.tensor(lens))
        graph.replay()
        assert dev.status() == 0
        assert torch.equal(kept.cpu(), ref.evict(w, lens, keep, 0, 0)[0]) and c.cache_len.tolist() == [keep, keep]
