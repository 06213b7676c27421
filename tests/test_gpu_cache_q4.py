"""The 4-bit cache on the GPU: commit and read back bit for bit, attention and its logarithms against the 64-bit form over the cache's
values."""
import numpy as np
import pytest
import torch

import paper_2505_21467_b200 as dlm
import q4_reference as ref
from helpers import Dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return Dev()


class Cache:
    """A 4-bit cache of random bytes (any byte is a value), guarded on both sides, with a copy of its bytes on the host."""

    def __init__(self, dev, NL, B, H, capacity, D, lens, seed):
        g = torch.Generator().manual_seed(seed)
        self.shape = (NL, B, H, capacity, D)
        x = {"k": torch.randn(NL, B, H, capacity, D, generator=g), "v": torch.randn(NL, B, H, capacity, D, generator=g)}
        x["k"][..., 5::16] *= 8
        self.host, self.gpu = {}, {}
        for n, t in x.items():
            self.host[n], self.host[n + "_scale"] = ref.pack(*ref.quantise(t.bfloat16()))
            for b, length in enumerate(lens):      # rows that nobody sees: the largest values there are
                self.host[n][:, b, :, length:], self.host[n + "_scale"][:, b, :, length:] = 255, 255
        for n, t in self.host.items():
            self.gpu[n] = dev.guarded(tuple(t.shape), torch.uint8, 0)
            self.gpu[n].copy_(t)
        self.cache_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.view = dlm.make_kv_cache_q4(self.gpu["k"], self.gpu["v"], self.gpu["k_scale"], self.gpu["v_scale"], self.cache_len)

    def values(self, n, layer):
        return ref.values(self.host[n][layer], self.host[n + "_scale"][layer])

    def check_bytes(self):
        for n, t in self.host.items():
            np.testing.assert_array_equal(self.gpu[n].cpu().numpy(), t.numpy(), err_msg=n)


def hard_rows(g, *shape):
    """bf16 rows with what quantisation can go wrong on: many magnitudes, ties, zeros, infinities, NaN, subnormals."""
    x = torch.randn(*shape, generator=g) * torch.exp2(torch.randint(-30, 20, shape[:-1] + (1,), generator=g).float())
    pick = torch.randint(0, 12, shape, generator=g)
    x = torch.where(pick == 0, torch.randint(-15, 16, shape, generator=g) / 2.0, x)          # halves: ties of small scales
    rows = torch.randint(0, 8, shape[:-1] + (1,), generator=g)
    x = torch.where(rows == 0, torch.randint(-15, 16, shape, generator=g) / 2.0 * torch.exp2(torch.randint(-4, 5, shape[:-1] + (1,), generator=g).float()), x)
    x = torch.where(rows == 1, torch.zeros_like(x), x)
    x = torch.where((rows == 2) & (pick == 1), torch.tensor(float("nan")), x)
    x = torch.where((rows == 3) & (pick == 1), torch.tensor(float("inf")), x)
    x = torch.where((rows == 3) & (pick == 2), torch.tensor(-float("inf")), x)
    x = torch.where(rows == 4, x * 1e-38, x)
    return x.bfloat16()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("NL,B,H,rows", [(1, 1, 1, 1), (3, 2, 2, 37), (2, 3, 4, 1000)])
def test_append_quantises_like_the_definition(dev, D, NL, B, H, rows):
    g = torch.Generator().manual_seed(100 + rows + D)
    capacity = (rows + 20) // 8 * 8
    lens = [int(torch.randint(0, capacity - rows + 1, (1,), generator=g)) for _ in range(B)]
    c = Cache(dev, NL, B, H, capacity, D, lens, 7)
    k, v = hard_rows(g, NL, B, H, rows, D), hard_rows(g, NL, B, H, rows, D)
    n_rows = torch.randint(0, rows + 1, (B,), generator=g, dtype=torch.int32)
    dlm.dlm_kv_cache_commit_q4(dev.ctx, c.view, k.cuda(), v.cuda(), rows, None, None, dlm.DLM_DST_APPEND, n_rows.cuda(), rows, 1, 0, NL)
    assert dev.status() == 0
    for name, t in (("k", k), ("v", v)):
        data, scale = ref.pack(*ref.quantise(t))
        for b in range(B):
            n, at = int(n_rows[b]), lens[b]
            c.host[name][:, b, :, at:at + n], c.host[name + "_scale"][:, b, :, at:at + n] = data[:, b, :, :n], scale[:, b, :, :n]
    c.check_bytes()
    assert c.cache_len.tolist() == [a + int(n) for a, n in zip(lens, n_rows)]


@pytest.mark.parametrize("D", [64, 128])
def test_scatter_layers_and_read_back(dev, D):
    g = torch.Generator().manual_seed(5)
    NL, B, H, capacity, L, R = 3, 2, 2, 72, 19, 7
    c = Cache(dev, NL, B, H, capacity, D, [11, 40], 8)
    k, v = hard_rows(g, 1, B, H, L, D), hard_rows(g, 1, B, H, L, D)
    src = torch.stack([torch.randperm(L, generator=g)[:R] for _ in range(B)]).int()
    dst = torch.stack([torch.randperm(capacity, generator=g)[:R] for _ in range(B)]).int()
    src[1, 2], dst[0, 3] = L, -1                            # one index out of range each: those rows are skipped
    dlm.dlm_kv_cache_commit_q4(dev.ctx, c.view, k.cuda(), v.cuda(), L, src.cuda(), dst.cuda(), dlm.DLM_DST_APPEND, None, R, 0, 1, 2)
    assert dev.status() == dlm.DLM_ERR_INDEX
    for name, t in (("k", k), ("v", v)):
        data, scale = ref.pack(*ref.quantise(t))
        for b in range(B):
            for r in range(R):
                if 0 <= src[b, r] < L and 0 <= dst[b, r] < capacity:
                    c.host[name][1, b, :, dst[b, r]], c.host[name + "_scale"][1, b, :, dst[b, r]] = data[0, b, :, src[b, r]], scale[0, b, :, src[b, r]]
    c.check_bytes()
    # read: rows in any order, a count per sequence, positions out of range
    pos = torch.randint(0, capacity, (B, 9), generator=g).int()
    n = torch.tensor([9, 4], dtype=torch.int32)
    ko, vo = (dev.guarded((2, B, H, 9, D), torch.bfloat16, 3.0) for _ in range(2))
    dlm.dlm_kv_cache_read_q4(dev.ctx, c.view, pos.cuda(), n.cuda(), 9, 1, 3, ko, vo)
    assert dev.status() == 0
    for name, got in (("k", ko), ("v", vo)):
        want = torch.full((2, B, H, 9, D), 3.0, dtype=torch.float64)
        for l in (1, 2):
            val = c.values(name, l)
            for b in range(B):
                want[l - 1, b, :, :n[b]] = val[b][:, pos[b, :n[b]].long()]
        assert torch.equal(got.cpu().double(), want)
    pos[0, 0] = capacity
    ko.fill_(3.0)
    dlm.dlm_kv_cache_read_q4(dev.ctx, c.view, pos.cuda(), torch.tensor([1, 10], dtype=torch.int32).cuda(), 9, 0, 3, *(torch.full((3, B, H, 9, D), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    assert dev.status() in (dlm.DLM_ERR_INDEX, dlm.DLM_ERR_CAPACITY)


@pytest.mark.parametrize("D", [64, 128])
def test_read_without_positions_and_the_window_mode(dev, D):
    g = torch.Generator().manual_seed(6)
    c = Cache(dev, 2, 2, 1, 40, D, [8, 21], 9)
    k, v = hard_rows(g, 2, 2, 1, 16, D), hard_rows(g, 2, 2, 1, 16, D)
    src = torch.tensor([[3, 15, 0], [1, 2, 9]], dtype=torch.int32)
    dlm.dlm_kv_cache_commit_q4(dev.ctx, c.view, k.cuda(), v.cuda(), 16, src.cuda(), None, dlm.DLM_DST_WINDOW, None, 3, 0, 0, 2)
    ko, vo = (dev.guarded((2, 2, 1, 40, D), torch.bfloat16, 3.0) for _ in range(2))
    dlm.dlm_kv_cache_read_q4(dev.ctx, c.view, None, None, 40, 0, 2, ko, vo)
    assert dev.status() == 0
    for name, got, new in (("k", ko, k), ("v", vo, v)):
        for b, at in enumerate((8, 21)):
            rows = at + src[b].long()
            assert torch.equal(got[:, b].cpu().double()[:, :, rows], ref.held(new)[:, b][:, :, src[b].long()])
    # too many rows for the capacity: nothing is written for that sequence
    before = {n: t.clone() for n, t in c.gpu.items()}
    c.cache_len.fill_(30)
    dlm.dlm_kv_cache_commit_q4(dev.ctx, c.view, k.cuda(), v.cuda(), 16, None, None, dlm.DLM_DST_APPEND, None, 16, 1, 0, 2)
    assert dev.status() == dlm.DLM_ERR_CAPACITY
    assert all(torch.equal(before[n], c.gpu[n]) for n in before) and c.cache_len.tolist() == [30, 30]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q4", [True, False])
def test_commits_of_more_items_than_a_wave_has_threads(dev, D, q4):
    """Both commit kernels: 4-bit rows against the definition, and the bf16 commit next to them as before."""
    g = torch.Generator().manual_seed(12)
    NL, B, H, rows = 4, 3, 4, 2111
    k, v = torch.randn(NL, B, H, rows, D, generator=g).bfloat16(), torch.randn(NL, B, H, rows, D, generator=g).bfloat16()
    if q4:
        c = Cache(dev, NL, B, H, 2112, D, [0] * B, 3)
        dlm.dlm_kv_cache_commit_q4(dev.ctx, c.view, k.cuda(), v.cuda(), rows, None, None, dlm.DLM_DST_APPEND, None, rows, 1, 0, NL)
        for name, t in (("k", k), ("v", v)):
            c.host[name][:, :, :, :rows], c.host[name + "_scale"][:, :, :, :rows] = ref.pack(*ref.quantise(t))
        assert dev.status() == 0
        c.check_bytes()
    else:
        ck, cv = (torch.zeros(NL, B, H, 2112, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        n = torch.zeros(B, dtype=torch.int32, device="cuda")
        dlm.dlm_kv_cache_commit(dev.ctx, dlm.make_kv_cache(ck, cv, n), k.cuda(), v.cuda(), rows, None, None, dlm.DLM_DST_APPEND, None, rows, 1, 0, NL)
        assert dev.status() == 0
        assert torch.equal(ck[:, :, :, :rows].cpu(), k) and torch.equal(cv[:, :, :, :rows].cpu(), v) and n.tolist() == [rows] * B


# --------------------------------------------------------------------------------------------------- attention

def attention_call(dev, c, q, kn, vn, q_len, layers=None, scale=0.0, lse=True):
    NL, B, H, capacity, D = c.shape
    lb, le = layers or (0, NL)
    Hq, L = q.shape[2], q.shape[3]
    out = dev.guarded(tuple(q.shape), torch.bfloat16, float("nan"))
    ls = dev.guarded(tuple(q.shape[:4]), torch.float32, float("nan")) if lse else None
    ws = dev.workspace(dlm.dlm_attn_workspace_bytes_q4(dev.ctx, c.view, le - lb, Hq, L))
    dlm.dlm_freecache_attn_step_q4(dev.ctx, c.view, lb, le, q, kn, vn, Hq, L, q_len, scale, 0, out, ls, ws)
    return out, ls


def inputs(NL, B, Hq, H, L, D, lq, seed):
    g = torch.Generator().manual_seed(seed)
    q, k, v = torch.randn(NL, B, Hq, L, D, generator=g), torch.randn(NL, B, H, L, D, generator=g), torch.randn(NL, B, H, L, D, generator=g)
    k[..., 5::16] *= 8
    for b, n in enumerate(lq):      # rows that take no part
        for t in (q, k, v):
            t[:, b, :, n:] = float("nan")
    return q.bfloat16(), k.bfloat16(), v.bfloat16()


def check_attention(c, q, kn, vn, lq, out, lse, layers=None, scale=None):
    """out: P and the result are rounded to bf16 (2^-8 each of sum p |v| and of the result); everything else is fp32: scores off by at
    most 2 D roundings of sum |q k| scale, which moves p by as much, and an exponential good to 2^-21.  lse: the same scores, and
    a logarithm and sums of fp32.  Weights below 2^-126 are no normal fp32 numbers and may be 0: of up to 2^12 keys with |v| < 2^4 they are
    2^-110 of an output."""
    lb, le = layers or (0, c.shape[0])
    D = q.shape[-1]
    for l in range(le - lb):
        w_out, w_lse, spread, size = ref.attention(c.values("k", lb + l), c.values("v", lb + l), c.cache_len.tolist(), q[l], kn[l], vn[l], lq, scale)
        off = size * 2 * D * 2.0 ** -24 + 2.0 ** -20
        tol = 2.0 ** -8 * (spread + w_out.abs()) * (1 + 2.0 ** -6) + 2 * off[..., None] * spread + 2.0 ** -110
        bad = (out[l].cpu().double() - w_out).abs() > tol
        assert not bool(bad.any()) and not bool(out[l].isnan().any()), (l, bad.nonzero()[:5], out[l].cpu()[bad][:5], w_out[bad][:5])
        if lse is not None:
            got = lse[l].cpu().double()
            assert torch.equal(got == -float("inf"), w_lse == -float("inf"))
            on = w_lse != -float("inf")
            lim = off + 2.0 ** -22 * (w_lse.abs() + 8)
            assert bool(((got - w_lse).abs() <= lim)[on].all()), float(((got - w_lse).abs() / lim)[on].max())


CASES = [
    # NL, B, Hq, H, D, L, cached rows, active rows
    (1, 1, 1, 1, 64, 1, [0], [1]),                                  # nothing cached, a single row
    (1, 1, 1, 1, 128, 1, [1], [1]),
    (1, 1, 4, 2, 64, 32, [256], [32]),
    (1, 1, 28, 4, 128, 32, [1024], [32]),                           # two M tiles, the second in part
    (2, 2, 8, 2, 128, 5, [63, 65], [5, 3]),
    (1, 3, 8, 8, 64, 17, [64, 0, 127], [17, 0, 1]),                 # an inactive sequence
    (3, 4, 4, 4, 128, 1, [200, 1, 128, 333], [1, 1, 0, 1]),         # single tokens
    (1, 2, 8, 2, 128, 77, [100, 31], [77, 64]),                     # several row chunks, fresh rows over a step
    (1, 1, 32, 1, 64, 40, [500], [40]),                             # a group of 32
    (2, 1, 4, 1, 128, 200, [0], [200]),                             # an initial pass
    (5, 3, 8, 4, 64, 9, [1000, 17, 640], [9, 9, 2]),                # more units than a block has, of odd lengths
    (40, 2, 4, 4, 128, 4, [90, 257], [4, 4]),                       # more units than SMs
    (1, 1, 2, 2, 128, 3, [5000], [3]),                              # few units, many steps: split over all SMs
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:6])))
def test_attention_matches_64_bits(dev, case):
    NL, B, Hq, H, D, L, lens, lq = case
    c = Cache(dev, NL, B, H, (max(lens) + 8) // 8 * 8, D, lens, 21)
    q, kn, vn = inputs(NL, B, Hq, H, L, D, lq, 22)
    q_len = None if lq == [L] * B else torch.tensor(lq, dtype=torch.int32, device="cuda")
    out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), q_len)
    assert dev.status() == 0
    check_attention(c, q, kn, vn, lq, out, lse)
    again, lse2 = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), q_len)
    assert dev.status() == 0
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse2)      # the same bits
    c.check_bytes()


def test_layer_range_scale_and_no_lse(dev):
    c = Cache(dev, 4, 2, 2, 128, 128, [100, 128], 31)
    q, kn, vn = inputs(2, 2, 4, 2, 11, 128, [11, 11], 32)
    out, _ = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None, layers=(1, 3), scale=0.03, lse=False)
    assert dev.status() == 0
    check_attention(c, q, kn, vn, [11, 11], out, None, layers=(1, 3), scale=0.03)


@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_grow_along_the_keys(dev, D):
    """The running maximum is raised by a lot many times: O is rescaled."""
    NL, B, H, L, C = 1, 1, 2, 6, 1500
    c = Cache(dev, NL, B, H, 1504, D, [C], 41)
    q, kn, vn = inputs(NL, B, 4, H, L, D, [L], 42)
    ramp = torch.linspace(0, 30, 1504)[None, None, None, :, None] * torch.ones(NL, B, H, 1504, D)
    ramp[..., 1::2] = 0.01
    data, scale = ref.pack(*ref.quantise(ramp.bfloat16()))
    q = q.abs()
    c.host["k"], c.host["k_scale"] = data, scale
    c.gpu["k"].copy_(data), c.gpu["k_scale"].copy_(scale)
    out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None)
    assert dev.status() == 0
    check_attention(c, q, kn, vn, [L], out, lse)


def test_lengths_out_of_range_are_clamped_and_reported(dev):
    c = Cache(dev, 1, 2, 2, 64, 64, [64, 64], 51)
    q, kn, vn = inputs(1, 2, 4, 2, 8, 64, [8, 8], 52)
    c.cache_len.copy_(torch.tensor([70, 64]))
    out, _ = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), torch.tensor([8, 9], dtype=torch.int32, device="cuda"))
    assert dev.status() == dlm.DLM_ERR_CAPACITY
    c.cache_len.copy_(torch.tensor([64, 64]))
    check_attention(c, q, kn, vn, [8, 8], out, None)


def test_workspace_is_checked(dev):
    c = Cache(dev, 1, 1, 1, 64, 64, [64], 61)
    q, kn, vn = inputs(1, 1, 1, 1, 8, 64, [8], 62)
    need = dlm.dlm_attn_workspace_bytes_q4(dev.ctx, c.view, 1, 1, 8)
    out = torch.empty_like(q, device="cuda")
    for ws in (torch.empty(need - 1, dtype=torch.uint8, device="cuda"), torch.empty(need + 16, dtype=torch.uint8, device="cuda")[16:]):
        with pytest.raises(dlm.DlmError) as e:
            dlm.dlm_freecache_attn_step_q4(dev.ctx, c.view, 0, 1, q.cuda(), kn.cuda(), vn.cuda(), 1, 8, None, 0.0, 0, out, None, ws)
        assert e.value.code == dlm.DLM_ERR_WORKSPACE


def test_a_captured_step_replays_on_new_lengths(dev):
    """commit and attention in one graph: lengths and contents are read when it is replayed."""
    NL, B, H, Hq, D, L = 2, 2, 2, 8, 128, 12
    c = Cache(dev, NL, B, H, 400, D, [0, 0], 71)
    q, kn, vn = (t.cuda() for t in inputs(NL, B, Hq, H, L, D, [L, L], 72))
    out, lse = torch.empty_like(q), torch.empty(NL, B, Hq, L, device="cuda")
    ws = torch.empty(dlm.dlm_attn_workspace_bytes_q4(dev.ctx, c.view, NL, Hq, L), dtype=torch.uint8, device="cuda")

    def step():
        dlm.dlm_freecache_attn_step_q4(dev.ctx, c.view, 0, NL, q, kn, vn, Hq, L, None, 0.0, 0, out, lse, ws)
        dlm.dlm_kv_cache_commit_q4(dev.ctx, c.view, kn, vn, L, None, None, dlm.DLM_DST_APPEND, None, L, 1, 0, NL)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        c.cache_len.zero_()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    for i in range(12):
        lens = [i * L] * B
        assert c.cache_len.tolist() == lens
        graph.replay()
        assert dev.status() == 0
        if i in (0, 1, 11):
            now = Cache.__new__(Cache)
            now.shape, now.host = c.shape, {n: t.cpu() for n, t in c.gpu.items()}
            now.cache_len = torch.tensor(lens)
            check_attention(now, q.cpu(), kn.cpu(), vn.cpu(), [L] * B, out, lse)


def test_the_kernels_give_up_instead_of_hanging(dev):
    """With no time to wait the first wait for data on its way gives up: an error code, and the context stays usable."""
    for L, Hq in ((4, 4), (32, 28)):
        c = Cache(dev, 2, 1, 4, 512, 128, [500], 81)
        q, kn, vn = inputs(2, 1, Hq, 4, L, 128, [L], 82)
        dlm.dlm_selftest_set_wait_limit(dev.ctx, 0)
        try:
            attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None)
            assert dev.status() == dlm.DLM_ERR_TIMEOUT
        finally:
            dlm.dlm_selftest_set_wait_limit(dev.ctx, 2_000_000_000)
        out, lse = attention_call(dev, c, q.cuda(), kn.cuda(), vn.cuda(), None)
        assert dev.status() == 0
        check_attention(c, q, kn, vn, [L], out, lse)
