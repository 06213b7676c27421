"""Plain 64-bit forms of the 4-bit cache, its attention, the rows' weights and eviction, written from the definitions in dlm.h, row by row
where that is clearer.  CPU tensors in, CPU tensors out."""
import math

import torch

GROUP, BIAS, LARGEST = 32, 20, 7.0 * 3840.0


def scale_value(byte):
    """What a scale byte stands for."""
    byte = int(byte)
    return (1 + (byte % 8) / 8) * 2.0 ** (byte // 8 - BIAS)


SCALES = torch.tensor([scale_value(b) for b in range(256)], dtype=torch.float64)


def quantise(x):
    """(n [..., D] in 1 .. 15, scale bytes [..., D / 32]) of values x."""
    x = x.double()
    x = torch.where(torch.isnan(x), torch.zeros_like(x), x.clamp(-LARGEST, LARGEST)).unflatten(-1, (-1, GROUP))
    amax = x.abs().amax(dim=-1)
    # the byte whose scale is nearest to amax / 7, compared without a division: the borders are half-way between neighbours, and
    # a tie goes to the byte of even m (neighbouring bytes differ by one, so to the even byte)
    border = 7 * (SCALES[1:] + SCALES[:-1]) / 2
    up_on_tie = torch.arange(1, 256) % 2 == 0
    byte = ((amax[..., None] > border) | ((amax[..., None] == border) & up_on_tie)).sum(dim=-1)
    s = SCALES[byte][..., None]
    # round(x / s), ties to even, likewise: n is the number of borders (k - 1/2) s that |x| reaches
    k = torch.arange(1, 8, dtype=torch.float64)
    half = (k - 0.5) * s[..., None]
    a = x.abs()[..., None]
    n = ((a > half) | ((a == half) & (k % 2 == 0))).sum(dim=-1)
    return (8 + torch.where(x < 0, -n, n)).flatten(-2), byte


def pack(n, byte):
    """The cache's bytes: uint8 [..., D / 2] and [..., D / 32]."""
    n = n.long().unflatten(-1, (-1, 8))
    word = sum(n[..., j] << (4 * (j // 2) + 16 * (j % 2)) for j in range(8))
    return torch.stack([(word >> (8 * i)) & 255 for i in range(4)], dim=-1).flatten(-2).to(torch.uint8), byte.to(torch.uint8)


def values(data, byte):
    """The values that bytes stand for, fp64 [..., D]."""
    b = data.long().unflatten(-1, (-1, 4))
    word = sum(b[..., i] << (8 * i) for i in range(4))
    n = torch.stack([(word >> (4 * (j // 2) + 16 * (j % 2))) & 15 for j in range(8)], dim=-1).flatten(-2)
    return ((n - 8).double().unflatten(-1, (-1, GROUP)) * SCALES[byte.long()][..., None]).flatten(-2)


def held(x):
    """The values that the cache holds for rows x."""
    return values(*pack(*quantise(x)))


def attention(k, v, cache_len, q, k_new, v_new, q_len, scale=None):
    """One layer.  k, v [B, Hkv, capacity, D] (values), q [B, Hq, L, D]; returns out, lse, and per output the sum of p |v| and per row the
    largest sum of |q_i k_i| * scale, which bound what rounding can do."""
    B, Hq, L, D = q.shape
    Hkv = k.shape[1]
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, spread = torch.zeros(B, Hq, L, D, dtype=torch.float64), torch.zeros(B, Hq, L, D, dtype=torch.float64)
    lse, size = torch.full((B, Hq, L), -math.inf, dtype=torch.float64), torch.zeros(B, Hq, L, dtype=torch.float64)
    for b in range(B):
        c, n = int(cache_len[b]), int(q_len[b])
        if n == 0:
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            keys = torch.cat([k[b, g, :c].double(), k_new[b, g, :n].double()])
            vals = torch.cat([v[b, g, :c].double(), v_new[b, g, :n].double()])
            rows = q[b, h, :n].double()
            z = rows @ keys.T * scale
            lse[b, h, :n] = torch.logsumexp(z, dim=-1)
            p = torch.softmax(z, dim=-1)
            out[b, h, :n], spread[b, h, :n] = p @ vals, p @ vals.abs()
            size[b, h, :n] = (rows.abs() @ keys.abs().T).amax(dim=-1) * scale
    return out, lse, spread, size


def weights(k, cache_len, q, lse, q_len, collected, decay, scale=None):
    """One layer: weight [B, Hkv, capacity] where visible (others nan), and the largest exponent's ingredients: max |s|, max |lse|."""
    B, Hq, L, D = q.shape
    Hkv = k.shape[1]
    scale = 1 / math.sqrt(D) if scale is None else scale
    w = torch.full(k.shape[:3], math.nan, dtype=torch.float64)
    most = 0.0
    for b in range(B):
        c, n = int(cache_len[b]), int(q_len[b])
        for g in range(Hkv):
            total = torch.zeros(c, dtype=torch.float64)
            for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                on = lse[b, h, :n] != -math.inf
                rows = q[b, h, :n][on].double()
                z = rows @ k[b, g, :c].double().T * scale
                total += (z - lse[b, h, :n][on].double()[:, None]).exp().sum(dim=0)
                if z.numel():
                    most = max(most, float((rows.abs() @ k[b, g, :c].double().abs().T).max() * scale + lse[b, h, :n][on].abs().max()))
            w[b, g, :c] = total + (decay * collected[b, g, :c].double() if collected is not None and decay != 0 else 0)
    return w, most


def evict(weight, cache_len, keep, protect_first, protect_last):
    """(kept_idx [..., keep], weight_out with nan where it is left as it was) of weight [NL, B, H, capacity]."""
    NL, B, H, C = weight.shape
    kept = torch.full((NL, B, H, keep), -1, dtype=torch.int32)
    out = torch.full(weight.shape, math.nan)
    for l in range(NL):
        for b in range(B):
            length = int(cache_len[b])
            n = min(keep, length)
            for h in range(H):
                w = weight[l, b, h].tolist()

                def rank(j):
                    if j < protect_first or j >= length - protect_last:
                        return (0, 0.0, j)
                    return (2, 0.0, j) if math.isnan(w[j]) else (1, -w[j], j)
                stay = set(sorted(range(length), key=rank)[:n])
                movers = iter(sorted(j for j in stay if j >= n))
                idx = [i if i in stay else next(movers) for i in range(n)]
                kept[l, b, h, :n] = torch.tensor(idx, dtype=torch.int32)
                out[l, b, h, :length] = 0.0
                out[l, b, h, :n] = weight[l, b, h][idx]
    return kept, out
