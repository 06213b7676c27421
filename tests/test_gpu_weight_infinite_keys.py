"""Attention weights of cached rows whose keys are not finite: a query row that takes no part contributes nothing to them, however many of such rows
stand beside the active ones in the products' tiles."""
import math

import pytest
import torch

import q4_reference as ref
from helpers import Dev
from test_gpu_cache_evict import Plain, accumulate
from test_gpu_cache_q4 import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return Dev()


def infinite_key_cache(dev, D, lens, capacity, rows, value, seed):
    """A bf16 cache whose `rows` have `value` in channel 3; its finite twin, with 0 there, is what .host keeps."""
    c = Plain(dev, 1, len(lens), 2, capacity, D, lens, seed)
    c.host["k"][..., 3] = torch.where(c.host["k"][..., 3].isnan(), c.host["k"][..., 3], torch.zeros((), dtype=torch.bfloat16))
    c.gpu["k"].copy_(c.host["k"])
    for r in rows:
        c.gpu["k"][..., r, 3] = value
    return c


# query heads a KV head, query rows, active ones: products of 16, 32, 128 columns, and of several chunks that stay (up to 256 rows) or go through
@pytest.mark.parametrize("g,L,n", [(1, 1, 1), (1, 15, 15), (1, 16, 16), (1, 17, 17), (2, 8, 3), (4, 32, 31), (1, 32, 30), (3, 60, 41), (2, 200, 200), (5, 77, 1)])
@pytest.mark.parametrize("D", [64, 128])
def test_a_key_of_minus_infinite_scores_keeps_what_it_has_collected(dev, D, g, L, n):
    """Every active row's score of the key is -infinity: no weight, so decay * collected, bit for bit.  The other keys' weights have the tolerance that
    test_weights_match_64_bits derives."""
    lens, lq, capacity = [300, 40], [n, max(1, n - 1)], 304
    rows = (0, 17, 39)
    c = infinite_key_cache(dev, D, lens, capacity, rows, -math.inf, 401)
    q, kn, vn = inputs(1, 2, 2 * g, 2, L, D, lq, 402)
    q[..., 3] = q[..., 3].abs() + 0.25                              # (inactive rows are NaN)
    lse = ref.attention(c.values("k", 0), c.values("v", 0), lens, q[0], kn[0], vn[0], lq)[1].float()[None]
    collected = torch.rand(1, 2, 2, capacity, generator=torch.Generator().manual_seed(403))
    weight = dev.guarded((1, 2, 2, capacity), torch.float32, -5.0)
    accumulate(dev, c, q.cuda(), lse.cuda(), torch.tensor(lq, dtype=torch.int32, device="cuda"), collected.cuda(), 0.5, weight)
    assert dev.status() == 0
    got = weight[0].cpu()
    want, most = ref.weights(c.values("k", 0), lens, q[0], lse[0], lq, collected[0], 0.5)
    for r in rows:
        assert torch.equal(got[:, :, r], 0.5 * collected[0, :, :, r])
        want[:, :, r] = 0.5 * collected[0, :, :, r].double()
    seen = ~want.isnan()
    rel = 2 * D * 2.0 ** -24 * most + 2.0 ** -22 * most + 2.0 ** -20 + g * L * 2.0 ** -24
    assert bool(((got.double() - want).abs() <= rel * want.abs() + 2.0 ** -23)[seen].all())
    assert bool((got[~seen] == -5.0).all())


@pytest.mark.parametrize("g,L", [(1, 1), (2, 20), (5, 77)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_keys_that_nobody_looks_at_keep_what_they_have_collected(dev, value, g, L):
    """Sequence 0 has no active rows, sequence 1 only rows that the attention step left out (lse = -infinity): whatever the key."""
    lens, lq, capacity, D = [130, 60], [0, L], 136, 128
    rows = (0, 5, 59)
    c = infinite_key_cache(dev, D, lens, capacity, rows, value, 411)
    q, _, _ = inputs(1, 2, 2 * g, 2, L, D, lq, 412)
    lse = torch.full((1, 2, 2 * g, L), -math.inf)
    collected = torch.rand(1, 2, 2, capacity, generator=torch.Generator().manual_seed(413))
    weight = dev.guarded((1, 2, 2, capacity), torch.float32, -5.0)
    accumulate(dev, c, q.cuda(), lse.cuda(), torch.tensor(lq, dtype=torch.int32, device="cuda"), collected.cuda(), 0.5, weight)
    assert dev.status() == 0
    for b, length in enumerate(lens):
        assert torch.equal(weight[0, b, :, :length].cpu(), 0.5 * collected[0, b, :, :length])
        assert bool((weight[0, b, :, length:] == -5.0).all())


@pytest.mark.parametrize("D", [64, 128])
def test_what_is_not_finite_by_the_formula_stays_so(dev, D):
    """A key whose scores are +infinite for some rows (-infinite for others) has an infinite weight, a key with a NaN a NaN; the other keys' weights
    are as without them."""
    lens, L, capacity = [200], 9, 200
    c = infinite_key_cache(dev, D, lens, capacity, (), 0.0, 421)
    clean = c.gpu["k"].clone()
    c.gpu["k"][0, 0, :, 7, 3], c.gpu["k"][0, 0, :, 70, 3], c.gpu["k"][0, 0, :, 150, 3] = math.inf, math.nan, -math.inf
    q, kn, vn = inputs(1, 1, 4, 2, L, D, [L], 422)
    q[..., 3] = q[..., 3].abs() + 0.25
    q[..., 1::2, 3] *= -1
    lse = ref.attention(c.values("k", 0), c.values("v", 0), lens, q[0], kn[0], vn[0], [L])[1].float()[None]
    lse[0, 0, 0, 2] = -math.inf                                     # a row that is left out
    q[0, 0, 0, 2] = math.nan
    weight, plain = (dev.guarded((1, 1, 2, capacity), torch.float32, 0.0) for _ in range(2))
    accumulate(dev, c, q.cuda(), lse.cuda(), None, None, 1.0, weight)
    c.gpu["k"].copy_(clean)
    accumulate(dev, c, q.cuda(), lse.cuda(), None, None, 1.0, plain)
    assert dev.status() == 0
    weight, plain = weight[0, 0].cpu(), plain[0, 0].cpu()
    assert bool((weight[:, 7] == math.inf).all()) and bool(weight[:, 70].isnan().all()) and bool((weight[:, 150] == math.inf).all())
    same = torch.ones(capacity, dtype=torch.bool)
    same[7] = same[70] = same[150] = False
    assert torch.equal(weight[:, same], plain[:, same])
