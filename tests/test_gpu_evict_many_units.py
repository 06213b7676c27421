"""Eviction where there is a unit for every SM, so that a block selects and moves its own rows: every size of block, one tile of weights and several."""
import math

import pytest
import torch

import paper_2505_21467_b200 as dlm
import q4_reference as ref
from helpers import Dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return Dev()


class OnDevice:
    """A cache of random bytes made on the device (any bytes can be moved)."""

    def __init__(self, dev, q4, NL, B, H, capacity, D, lens, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        parts = {"k": D // 2, "v": D // 2, "k_scale": D // 32, "v_scale": D // 32} if q4 else {"k": 2 * D, "v": 2 * D}
        self.gpu = {}
        for n, width in parts.items():
            t = dev.guarded((NL, B, H, capacity, width), torch.uint8, 0)
            t.random_(0, 256, generator=g)
            self.gpu[n] = t
        self.cache_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        if q4:
            self.view = dlm.make_kv_cache_q4(*(self.gpu[n] for n in ("k", "v", "k_scale", "v_scale")), self.cache_len)
        else:
            self.view = dlm.make_kv_cache(self.gpu["k"].view(torch.bfloat16), self.gpu["v"].view(torch.bfloat16), self.cache_len)
        self.q4 = q4


def call(dev, c, weight, keep, first, last, out):
    kept = dev.guarded(tuple(weight.shape[:3]) + (keep,), torch.int32, -7)
    f = dlm.dlm_kv_cache_evict_q4 if c.q4 else dlm.dlm_kv_cache_evict
    f(dev.ctx, c.view, weight, keep, first, last, kept, out)
    return kept


def what_stays(weight, length, keep, first, last):
    """[units, length] truth values: the definition by two stable sorts; NaN below every number, protected rows first."""
    w = weight.reshape(-1, weight.shape[-1])[:, :length]
    j = torch.arange(length, device=w.device)
    order = torch.where(w.isnan(), torch.full_like(w, -math.inf), w).argsort(dim=-1, descending=True, stable=True)
    kind = torch.where((j < first) | (j >= length - last), 0, torch.where(w.isnan(), 2, 1))
    order = order.gather(-1, kind.gather(-1, order).argsort(dim=-1, stable=True))
    return torch.zeros_like(kind, dtype=torch.bool).scatter_(-1, order[:, :min(keep, length)], True)


def check(dev, q4, shape, lens, keep, first, last, weight, mode, seed):
    NL, B, H, capacity, D = shape
    c = OnDevice(dev, q4, NL, B, H, capacity, D, lens, seed)
    before = {n: t.clone() for n, t in c.gpu.items()}
    w = dev.guarded(tuple(weight.shape), torch.float32, 0.0)
    w.copy_(weight)
    out = {"in_place": w, "apart": dev.guarded(tuple(weight.shape), torch.float32, -3.0), "none": None}[mode]
    kept = call(dev, c, w, keep, first, last, out)
    assert dev.status() == 0
    assert c.cache_len.tolist() == [min(n, keep) for n in lens]
    for b, length in enumerate(lens):
        n = min(keep, length)
        stay = what_stays(weight[:, b], length, keep, first, last)
        idx = torch.arange(n, device="cuda").expand(stay.shape[0], n).clone()
        idx[~stay[:, :n]] = torch.nonzero(stay[:, n:])[:, 1] + n                # units, then rows, both ascending: the k-th mover to the k-th hole
        got = kept[:, b].reshape(-1, keep)
        assert torch.equal(got[:, :n].long(), idx) and bool((got[:, n:] == -1).all())
        if b == 0:
            # the sorts above against the definition row by row
            u = weight[-1:, b:b + 1, -1:, :].cpu()
            assert torch.equal(ref.evict(u, [length], keep, first, last)[0].flatten()[:n].long(), idx[-1].cpu())
        if out is not None:
            o, src = out[:, b].reshape(-1, capacity), weight[:, b].reshape(-1, capacity)
            same = lambda x, y: torch.equal(x.nan_to_num(7.5), y.nan_to_num(7.5))
            assert same(o[:, :n], src.gather(-1, idx)) and bool((o[:, n:length] == 0).all())
            assert same(o[:, length:], src[:, length:] if mode == "in_place" else torch.full_like(o[:, length:], -3.0))
        for name, t in before.items():
            rows, now = t[:, b].reshape(-1, capacity, t.shape[-1]), c.gpu[name][:, b].reshape(-1, capacity, t.shape[-1])
            assert torch.equal(now[:, :n], rows.gather(1, idx[..., None].expand(-1, -1, t.shape[-1]))), name
            assert torch.equal(now[:, n:], rows[:, n:]), name


@pytest.mark.parametrize("q4", [True, False])
@pytest.mark.parametrize("mode", ["in_place", "apart", "none"])
@pytest.mark.parametrize("capacity", [608, 1024, 3000, 6000, 12000, 17000, 40000])
def test_blocks_that_move_their_own_rows(dev, q4, mode, capacity):
    """160 units of two lengths; weights that differ, and weights with ties, zeros of both signs, infinities and NaN."""
    NL, B, H, D = 10, 2, 8, 64
    lens = [capacity - 7, capacity * 2 // 3]
    g = torch.Generator(device="cuda").manual_seed(901)
    for ties, (keep, first, last) in ((False, (capacity // 2, 4, 32)), (True, (capacity * 3 // 5, 0, 1))):
        weight = torch.rand(NL, B, H, capacity, device="cuda", generator=g)
        if ties:
            weight = (weight * 5).floor() * 0.5 - 1.0
            pick = torch.rand(weight.shape, device="cuda", generator=g)
            for value, share in ((-0.0, 0.05), (math.nan, 0.08), (math.inf, 0.11), (-math.inf, 0.14)):
                weight = torch.where((pick < share) & (pick >= share - 0.03), torch.full_like(weight, value), weight)
        check(dev, q4, (NL, B, H, capacity, D), lens, keep, first, last, weight, mode, 902)


@pytest.mark.parametrize("units", [(1, 1, 147), (1, 1, 148), (1, 149, 1), (37, 2, 2)])
def test_numbers_of_units_beside_the_number_of_sms(dev, units):
    NL, B, H = units
    lens = [(200 + 13 * b) % 301 for b in range(B)]
    weight = torch.rand(NL, B, H, 304, device="cuda", generator=torch.Generator(device="cuda").manual_seed(911))
    check(dev, True, (NL, B, H, 304, 128), lens, 100, 3, 9, weight, "apart", 912)


def test_calls_without_a_pause_set_the_lengths_each_time(dev):
    """The last block to read a sequence's length sets the new one: many evictions in a row, each of what the one before has left."""
    NL, B, H, capacity = 20, 2, 4, 512
    c = OnDevice(dev, True, NL, B, H, capacity, 64, [500, 130], 921)
    weight = torch.rand(NL, B, H, capacity, device="cuda", generator=torch.Generator(device="cuda").manual_seed(922))
    want, lens, sets = weight.clone(), [500, 130], []
    for keep in range(450, 0, -50):
        kept = torch.empty(NL, B, H, keep, dtype=torch.int32, device="cuda")
        dlm.dlm_kv_cache_evict_q4(dev.ctx, c.view, weight, keep, 0, 2, kept, weight)
        sets.append((keep, kept))
    assert dev.status() == 0 and c.cache_len.tolist() == [50, 50]
    for keep, kept in sets:
        for b in range(B):
            n = min(keep, lens[b])
            stay = what_stays(want[:, b], lens[b], keep, 0, 2)
            idx = torch.arange(n, device="cuda").expand(stay.shape[0], n).clone()
            idx[~stay[:, :n]] = torch.nonzero(stay[:, n:])[:, 1] + n
            assert torch.equal(kept[:, b].reshape(-1, keep)[:, :n].long(), idx), (keep, b)
            flat = want[:, b].reshape(-1, capacity)
            new = flat.clone()
            new[:, :n], new[:, n:lens[b]] = flat.gather(-1, idx), 0
            want[:, b] = new.view(NL, H, capacity)
            lens[b] = n
    assert torch.equal(weight, want)
