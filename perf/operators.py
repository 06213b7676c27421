"""What a program that serves a diffusion language model asks of a 4-bit K/V cache and of a cache that throws rows out, as
measurable cases.

Four kinds of pass:

  commit   K/V rows go into the 4-bit cache (a prompt's, or the rows chosen in a denoising step) and are read back as bf16.
  attn     attention of the active window over [4-bit cache ; fresh rows], of one layer or of all layers in one call.
  weight   per cached row, the attention weight that the window's query rows give it, added to what it has collected; the cache in
           bf16 or in 4 bits.
  evict    of every (layer, sequence, KV head) the rows of largest weight are kept and brought to the front; bf16 or 4 bits.

A row of the 4-bit cache is groups of 32 consecutive values, value = (n - 8) * s: n of 4 bits, s a byte eeeeemmm that stands
for (1 + m / 8) * 2 ** (e - 20).  Eight consecutive values are a 32-bit word, value j in bits 4 * (j / 2) .. + 3 of its lower half
(j even) or upper half (j odd).

Values: queries and V rows N(0, 1); K rows N(0, 1) with one channel in 16 eight times as large, as key channels are.
"""
import math

import torch

own = False

DEVICE = "cuda"
GROUP = 32                # values per scale
BIAS = 20                 # of a scale's exponent
LARGEST = 7.0 * 3840.0    # the largest value that the format holds

DREAM = dict(n_q_heads=28, n_kv_heads=4, head_dim=128)
LLADA = dict(n_q_heads=32, n_kv_heads=32, head_dim=128)
TINY = dict(n_q_heads=4, n_kv_heads=2, head_dim=64)
SMALL = dict(n_q_heads=8, n_kv_heads=2, head_dim=128)
SMALL_MHA = dict(n_q_heads=8, n_kv_heads=8, head_dim=64)
MODELS = [DREAM, LLADA, TINY, SMALL, SMALL_MHA]


def listed():
    return [
        # the rows of the 4 positions chosen in a denoising step, staged at their slots in all 28 layers
        dict(name="commit_chosen", kind="commit", layers=28, batch=1, cache=1024, rows=4, block=32, scatter=True, ragged=False, **DREAM),
        # prompts of 8 sequences of different lengths appended to an empty cache
        dict(name="commit_prompts", kind="commit", layers=28, batch=8, cache=0, rows=1024, block=1024, scatter=False, ragged=True, **DREAM),
        # the smallest attention call
        dict(name="attn_tiny", kind="attn", layers=1, batch=1, block=32, cache=256, ragged=False, **TINY),
        # one layer of interactive decoding: a block of 32 behind a prompt of 1024
        dict(name="attn_layer", kind="attn", layers=1, batch=1, block=32, cache=1024, ragged=False, **DREAM),
        # single tokens of 8 sequences of different lengths, multi-head
        dict(name="attn_token", kind="attn", layers=1, batch=8, block=1, cache=4001, ragged=True, **LLADA),
        # a multi-head stack, 4 sequences, block 64, prompt 2048, 32 layers in one call
        dict(name="attn_stack", kind="attn", layers=32, batch=4, block=64, cache=2048, ragged=False, **LLADA),
        # long context, cache length off the tile grid, 28 layers in one call
        dict(name="attn_long", kind="attn", layers=28, batch=1, block=32, cache=16301, ragged=False, **DREAM),
        # weights of one layer's cached rows after its attention
        dict(name="weight_layer", kind="weight", bits=4, layers=1, batch=1, block=32, cache=1024, ragged=False, **DREAM),
        # weights of a long context's rows in all layers, bf16 cache
        dict(name="weight_long", kind="weight", bits=16, layers=28, batch=1, block=32, cache=16301, ragged=False, **DREAM),
        # weights in a 4-bit multi-head stack
        dict(name="weight_stack", kind="weight", bits=4, layers=32, batch=4, block=64, cache=2048, ragged=False, **LLADA),
        # half of a long context thrown out, 4 bits, all layers
        dict(name="evict_long", kind="evict", bits=4, layers=28, batch=1, cache=16301, keep=8192, first=4, last=32, ragged=False, **DREAM),
        # 8 sequences of different lengths brought to 700 rows, bf16
        dict(name="evict_batch8", kind="evict", bits=16, layers=28, batch=8, cache=1152, keep=700, first=0, last=64, ragged=True, **DREAM),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("commit", "attn", "weight", "evict")}
    while True:
        c = _draw_any(rng)
        if _cost(c) <= most[c["kind"]] and _plain_bytes(c) <= 12e9:
            return c


def _draw_any(rng):
    kind = rng.choice(["commit", "attn", "attn", "weight", "evict"])
    model = rng.choice(MODELS)
    batch, layers = _log_int(rng, 1, 8), _log_int(rng, 1, 32)
    ragged = batch > 1 and rng.random() < 0.5
    if kind == "commit":
        scatter = rng.random() < 0.5
        rows = _log_int(rng, 1, 64 if scatter else 3000)
        return dict(kind=kind, layers=layers, batch=batch, cache=_log_int(rng, 1, 4096), rows=rows,
                    block=rows + (rng.randint(0, 64) if scatter else 0), scatter=scatter, ragged=ragged, **model)
    if kind == "evict":
        cache = _log_int(rng, 16, 20000)
        keep = max(1, int(cache * rng.uniform(0.2, 0.95)))
        return dict(kind=kind, bits=rng.choice([4, 16]), layers=layers, batch=batch, cache=cache, keep=keep,
                    first=rng.randint(0, keep // 4), last=rng.randint(0, keep // 4), ragged=ragged, **model)
    c = dict(kind=kind, layers=layers, batch=batch, block=_log_int(rng, 1, 512), cache=_log_int(rng, 1, 20000), ragged=ragged, **model)
    if kind == "weight":
        c["bits"] = rng.choice([4, 16])
    return c


# ------------------------------------------------------------------------------------------------ sizes of a case

def _spread(n, batch, ragged):
    return [max(1, n - (b * 53) % max(2, n // 4)) if ragged else n for b in range(batch)]


def _lengths(case):
    """(cache_len[b], q_len[b]) of an attention or weight case."""
    return _spread(case["cache"], case["batch"], case["ragged"]), _spread(case["block"], case["batch"], case["ragged"])


def _n_rows(case):
    return _spread(case["rows"], case["batch"], case["ragged"])


def _bits(case):
    return 16.0 if case.get("bits", 4) == 16 else 4.0 + 8.0 / GROUP


def work(case):
    Hq, Hkv, D = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    B, nl = case["batch"], case["layers"]
    row = 2 * Hkv * D * _bits(case) / 8          # bytes of a cached row of a layer, K and V
    if case["kind"] == "commit":
        n = sum(_n_rows(case))
        return {"bytes": int(nl * n * (2 * 2 * 2 * Hkv * D + 2 * row)), "flops": nl * n * 2 * Hkv * D * 6}
    if case["kind"] == "evict":
        lens = _spread(case["cache"], B, case["ragged"])
        kept = [min(case["keep"], n) for n in lens]
        moved = sum(k * (1 - k / n) for k, n in zip(kept, lens))     # of rows whose weights are in no order
        small = nl * Hkv * (4 * sum(lens) + 4 * B * case["keep"] + 4 * sum(lens))   # weights, kept rows, weights of the kept
        return {"bytes": int(2 * nl * moved * row + small), "flops": nl * Hkv * sum(lens) * 4}
    lc, lq = _lengths(case)
    q_rows, pairs = sum(lq), sum(c * q for c, q in zip(lc, lq))
    if case["kind"] == "weight":
        return {"bytes": int(nl * (row / 2 * sum(lc) + 2 * Hq * D * q_rows + 4 * Hq * q_rows + 2 * 4 * Hkv * sum(lc))),
                "flops": nl * Hq * pairs * (2 * D + 3)}
    all_pairs = sum(q * (c + q) for c, q in zip(lc, lq))
    return {"bytes": int(nl * (row * sum(lc) + 2 * 2 * Hkv * D * q_rows + 2 * Hq * D * (q_rows + B * case["block"]) + 4 * Hq * B * case["block"])),
            "flops": nl * Hq * all_pairs * 4 * D}


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.6e15)


def _plain_bytes(case):
    """About what the plain form holds at a time."""
    B, nl, D = case["batch"], case["layers"], case["head_dim"]
    values = nl * B * case["n_kv_heads"] * D * (case["cache"] + case.get("rows", 0) + case.get("block", 0))
    scores = nl * B * case["n_q_heads"] * case.get("block", 0) * (case["cache"] + case.get("block", 0)) if case["kind"] in ("attn", "weight") else 0
    return 2 * 4 * values + 2 * 4 * scores


# ------------------------------------------------------------------------------------------------ the 4-bit rows

def _scale_of(byte):
    return (((byte.int() << 4) + ((127 - BIAS) << 7)) << 16).view(torch.float32)


def _pack(x):
    """Rows [..., D] -> (4-bit values uint8 [..., D / 2], scales uint8 [..., D / GROUP])."""
    g = x.float().clamp(-LARGEST, LARGEST).unflatten(-1, (-1, GROUP))
    amax = g.abs().amax(dim=-1)
    t = (amax / torch.full_like(amax, 7.0)).view(torch.int32)     # (by a number, torch multiplies with its reciprocal: borders move)
    byte = (((t + 0x7FFFF + ((t >> 20) & 1)) >> 20) - ((127 - BIAS) << 3)).clamp(0, 255)
    n = (torch.round(g / _scale_of(byte)[..., None]) + 8).to(torch.int32)
    n = n.flatten(-2).unflatten(-1, (-1, 4, 2)).transpose(-1, -2).flatten(-3)       # values 0 2 4 6 1 3 5 7 of each word
    return (n[..., 0::2] | (n[..., 1::2] << 4)).to(torch.uint8), byte.to(torch.uint8)


def _unpack(data, byte):
    """The values, fp32."""
    n = torch.stack([data & 15, data >> 4], dim=-1).flatten(-2).unflatten(-1, (-1, 2, 4)).transpose(-1, -2).flatten(-3)
    return ((n.float() - 8.0).unflatten(-1, (-1, GROUP)) * _scale_of(byte)[..., None]).flatten(-2)


# ------------------------------------------------------------------------------------------------ state

_context = None


def _ctx():
    """The process's library context, created once."""
    global _context
    if _context is None:
        import paper_2505_21467_b200 as dlm
        _context = dlm.dlm_create(torch.cuda.current_device())
    return _context


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _empty(*shape, dtype):
    return torch.empty(*shape, dtype=dtype, device=DEVICE)


def _rows(g, *shape, keys=False):
    t = torch.empty(*shape, dtype=torch.bfloat16, device=DEVICE).normal_(0.0, 1.0, generator=g)
    if keys:
        t[..., 5::16] *= 8
    return t


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    s = dict(case)
    B, nl, Hq, Hkv, D, C = case["batch"], case["layers"], case["n_q_heads"], case["n_kv_heads"], case["head_dim"], case["cache"]
    s["capacity"] = (C + case.get("block", 0) + 15) // 16 * 16
    if case.get("bits", 4) == 4:
        for x in ("k", "v"):
            s[x + "_data"] = _empty(nl, B, Hkv, s["capacity"], D // 2, dtype=torch.uint8)
            s[x + "_scale"] = _empty(nl, B, Hkv, s["capacity"], D // GROUP, dtype=torch.uint8)
            for l in range(nl):
                s[x + "_data"][l], s[x + "_scale"][l] = _pack(_rows(g, B, Hkv, s["capacity"], D, keys=x == "k"))
    else:
        s["k_cache"], s["v_cache"] = _rows(g, nl, B, Hkv, s["capacity"], D, keys=True), _rows(g, nl, B, Hkv, s["capacity"], D)
    if case["kind"] == "commit":
        _prepare_commit(s, g)
    elif case["kind"] == "evict":
        _prepare_evict(s, g)
    else:
        lc, lq = _lengths(case)
        L = case["block"]
        s["cache_len"], s["hint"] = _ints(lc), max(lc)
        s["q_len"] = _ints(lq) if case["ragged"] else None
        s["q"] = _rows(g, nl, B, Hq, L, D)
        s["k_new"], s["v_new"] = _rows(g, nl, B, Hkv, L, D, keys=True), _rows(g, nl, B, Hkv, L, D)
        s["out"] = _empty(nl, B, Hq, L, D, dtype=torch.bfloat16)
        s["lse"] = _empty(nl, B, Hq, L, dtype=torch.float32)
        if case["kind"] == "weight":      # what the attention step left, and what the rows had collected before it
            for l in range(nl):
                s["lse"][l:l + 1] = _log_sums(_scores(s, slice(l, l + 1))).view(1, B, Hq, L)
            s["collected"] = torch.rand(nl, B, Hkv, s["capacity"], generator=g, device=DEVICE)
            s["weight"] = s["collected"].clone()
    if own:
        _prepare_handles(s)
    return s


def _prepare_commit(s, g):
    B, nl, Hkv, D, L, R = s["batch"], s["layers"], s["n_kv_heads"], s["head_dim"], s["block"], s["rows"]
    s["k_new"], s["v_new"] = _rows(g, nl, B, Hkv, L, D, keys=True), _rows(g, nl, B, Hkv, L, D)
    s["n_rows"] = _ints(_n_rows(s)) if s["ragged"] else None
    s["cache_len"] = _ints([s["cache"]] * B)
    s["src_idx"] = torch.rand(B, L, generator=g, device=DEVICE).argsort(dim=1)[:, :R].sort(dim=1).values.int().contiguous() if s["scatter"] else None
    from_row = s["src_idx"] if s["scatter"] else torch.arange(R, device=DEVICE, dtype=torch.int32).expand(B, R)
    s["positions"] = (s["cache_len"][:, None] + from_row).int().contiguous()
    # rows beyond a sequence's count stay what they are
    s["k_out"], s["v_out"] = torch.zeros(nl, B, Hkv, R, D, dtype=torch.bfloat16, device=DEVICE), torch.zeros(nl, B, Hkv, R, D, dtype=torch.bfloat16, device=DEVICE)


def _prepare_evict(s, g):
    B, nl, Hkv = s["batch"], s["layers"], s["n_kv_heads"]
    s["lens"] = _ints(_spread(s["cache"], B, s["ragged"]))
    s["cache_len"] = s["lens"].clone()
    # collected weights are skewed: a few rows have most of them
    s["weight"] = torch.rand(nl, B, Hkv, s["capacity"], generator=g, device=DEVICE).clamp_(min=1e-6).reciprocal_().sqrt_()
    s["weight_out"] = torch.zeros(nl, B, Hkv, s["capacity"], dtype=torch.float32, device=DEVICE)
    s["kept_idx"] = _empty(nl, B, Hkv, s["keep"], dtype=torch.int32)


def _prepare_handles(s):
    import paper_2505_21467_b200 as dlm
    s["ctx"] = _ctx()
    if s.get("bits", 4) == 4:
        s["handle"] = dlm.make_kv_cache_q4(s["k_data"], s["v_data"], s["k_scale"], s["v_scale"], s["cache_len"])
    else:
        s["handle"] = dlm.make_kv_cache(s["k_cache"], s["v_cache"], s["cache_len"])
    if s["kind"] == "attn":
        n = dlm.dlm_attn_workspace_bytes_q4(s["ctx"], s["handle"], s["layers"], s["n_q_heads"], s["block"])
        s["workspace"] = _empty(max(int(n), 256), dtype=torch.uint8)


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    return {"commit": _run_commit, "attn": _run_attn, "weight": _run_weight, "evict": _run_evict}[s["kind"]](s)


def _run_commit(s):
    nl, R = s["layers"], s["rows"]
    if own:
        import paper_2505_21467_b200 as dlm
        dlm.dlm_kv_cache_commit_q4(s["ctx"], s["handle"], s["k_new"], s["v_new"], s["block"], s["src_idx"], None,
                                   dlm.DLM_DST_WINDOW if s["scatter"] else dlm.DLM_DST_APPEND, s["n_rows"], R, 0, 0, nl)
        dlm.dlm_kv_cache_read_q4(s["ctx"], s["handle"], s["positions"], s["n_rows"], R, 0, nl, s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    B, Hkv, D = s["batch"], s["n_kv_heads"], s["head_dim"]
    at = s["positions"].long()[None, :, None, :, None].expand(nl, B, Hkv, R, 1)
    written = None if s["n_rows"] is None else (torch.arange(R, device=DEVICE) < s["n_rows"][:, None])[None, :, None, :, None]
    res = {}
    for x in ("k", "v"):
        new = s[x + "_new"]
        if s["scatter"]:
            new = new.gather(3, s["src_idx"].long()[None, :, None, :, None].expand(nl, B, Hkv, R, D))
        for part, t in zip((s[x + "_data"], s[x + "_scale"]), _pack(new)):
            i = at.expand(-1, -1, -1, -1, part.shape[-1])
            part.scatter_(3, i, t if written is None else torch.where(written, t, part.gather(3, i)))
        back = _unpack(s[x + "_data"].gather(3, at.expand(-1, -1, -1, -1, D // 2)),
                       s[x + "_scale"].gather(3, at.expand(-1, -1, -1, -1, D // GROUP))).to(torch.bfloat16)
        res[x] = back if written is None else torch.where(written, back, s[x + "_out"])
    return res


def _masks(s):
    """Which keys [B, C + L] and query rows [B, L] take part; C the rows that the longest cache has."""
    C, L = s["cache"], s["block"]
    lq = s["q_len"] if s["q_len"] is not None else torch.full_like(s["cache_len"], L)
    rows = torch.arange(L, device=DEVICE) < lq[:, None]
    return torch.cat([torch.arange(C, device=DEVICE) < s["cache_len"][:, None], rows], dim=1), rows


def _values(s, x, layers):
    """K or V of all keys, fp32 [layers, B, Hkv, C + L, D]."""
    C = s["cache"]
    if s.get("bits", 4) == 4:
        c = _unpack(s[x + "_data"][layers, :, :, :C], s[x + "_scale"][layers, :, :, :C])
    else:
        c = s[x + "_cache"][layers, :, :, :C].float()
    return torch.cat([c, s[x + "_new"][layers].float()], dim=3)


def _scores(s, layers):
    """Scaled scores, fp32 [layers, B, Hkv, group * L, C + L], -inf where a key or a query row takes no part."""
    Hkv, D = s["n_kv_heads"], s["head_dim"]
    keys, rows = _masks(s)
    q = s["q"][layers].float().unflatten(2, (Hkv, -1)).flatten(3, 4)
    z = (q @ _values(s, "k", layers).transpose(-1, -2)).mul_(D ** -0.5)
    on = rows.repeat(1, s["n_q_heads"] // Hkv)[:, :, None] & keys[:, None, :]
    return z.masked_fill_(~on[None, :, None], -math.inf)


def _log_sums(z):
    """log sum exp of the scores, fp32 [layers, B, Hq, L] flattened over the heads' rows."""
    m = z.amax(dim=-1, keepdim=True)
    safe = torch.where(m == -math.inf, torch.zeros_like(m), m)
    total = (z - safe).exp_().sum(dim=-1)
    lse = total.log().add_(safe[..., 0])
    return lse


def _run_attn(s):
    nl, Hq, L = s["layers"], s["n_q_heads"], s["block"]
    if own:
        import paper_2505_21467_b200 as dlm
        dlm.dlm_freecache_attn_step_q4(s["ctx"], s["handle"], 0, nl, s["q"], s["k_new"], s["v_new"], Hq, L, s["q_len"], 0.0, s["hint"],
                                       s["out"], s["lse"], s["workspace"])
        return {"out": s["out"], "lse": s["lse"]}
    every = slice(None)
    z = _scores(s, every)
    m = z.amax(dim=-1, keepdim=True)
    p = (z - torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    lse = (total.log() + m)[..., 0]
    out = (p @ _values(s, "v", every)) / torch.where(total == 0, torch.ones_like(total), total)
    shape = (nl, s["batch"], Hq, L)
    return {"out": out.to(torch.bfloat16).view(*shape, -1), "lse": lse.view(shape)}


DECAY = 0.75


def _run_weight(s):
    nl, Hq, L = s["layers"], s["n_q_heads"], s["block"]
    if own:
        import paper_2505_21467_b200 as dlm
        call = dlm.dlm_cache_weight_accumulate_q4 if s["bits"] == 4 else dlm.dlm_cache_weight_accumulate
        call(s["ctx"], s["handle"], 0, nl, s["q"], s["lse"], Hq, L, s["q_len"], 0.0, s["hint"], s["collected"], DECAY, s["weight"])
        return {"weight": s["weight"]}
    C, Hkv = s["cache"], s["n_kv_heads"]
    z = _scores(s, slice(None))[..., :C]
    lse = s["lse"].view(*z.shape[:-1], 1)
    got = (z - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)).exp_().sum(dim=-2)
    visible = (torch.arange(C, device=DEVICE) < s["cache_len"][:, None])[None, :, None]
    w = s["weight"][..., :C]
    w.copy_(torch.where(visible, DECAY * s["collected"][..., :C] + got, w))
    return {"weight": s["weight"]}


def _run_evict(s):
    s["cache_len"].copy_(s["lens"])
    parts = ["k_data", "k_scale", "v_data", "v_scale"] if s["bits"] == 4 else ["k_cache", "v_cache"]
    if own:
        import paper_2505_21467_b200 as dlm
        call = dlm.dlm_kv_cache_evict_q4 if s["bits"] == 4 else dlm.dlm_kv_cache_evict
        call(s["ctx"], s["handle"], s["weight"], s["keep"], s["first"], s["last"], s["kept_idx"], s["weight_out"])
    else:
        C, K = s["cache"], s["keep"]
        j = torch.arange(C, device=DEVICE)
        lens = s["lens"][:, None].long()                                                     # [B, 1]
        n = lens.clamp(max=K)
        w = s["weight"][..., :C]
        protected = ((j < s["first"]) | (j >= lens - s["last"]))[None, :, None]
        rank = torch.where((j < lens)[None, :, None], torch.where(protected, torch.full_like(w, math.inf), w), torch.full_like(w, -math.inf))
        order = rank.argsort(dim=-1, descending=True, stable=True)
        kept = torch.zeros_like(w, dtype=torch.bool).scatter_(-1, order, (j < n)[None, :, None].expand_as(w))
        front = (j < n)[None, :, None]
        mover, hole = kept & ~front, ~kept & front
        to = torch.where(mover, mover.cumsum(-1) - 1, torch.full_like(order, C))              # k-th mover -> entry k
        movers = torch.zeros(*w.shape[:-1], C + 1, dtype=torch.long, device=DEVICE).scatter_(-1, to, j.expand_as(order))
        src = torch.where(hole, movers.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)), j.expand_as(order))[..., :K]
        live = (j[:K] < n)[None, :, None]
        s["kept_idx"] = torch.where(live, src, torch.full_like(src, -1)).int()
        at = torch.where(live, src, j[:K].expand_as(src))
        out = s["weight_out"]
        out[..., :C] = torch.where((j < lens)[None, :, None], torch.zeros_like(w), out[..., :C])
        out[..., :K] = torch.where(live, s["weight"].gather(-1, at), out[..., :K])
        for x in parts:
            t = s[x]
            t[..., :K, :] = t.gather(3, at[..., None].expand(-1, -1, -1, -1, t.shape[-1]))
        s["cache_len"].copy_(n[:, 0])
    # the rows are moved, not computed: the 4-bit cache's come as they are held
    return {"kept_idx": s["kept_idx"], "weight_out": s["weight_out"], "cache_len": s["cache_len"], **{x: s[x] for x in parts}}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _values64(s, x, l):
    if s.get("bits", 4) == 16:
        return s[x + "_cache"][l, :, :, :s["cache"]].double()
    word = s[x + "_data"][l, :, :, :s["cache"]].long().unflatten(-1, (-1, 4))
    word = word[..., 0] + word[..., 1] * 2 ** 8 + word[..., 2] * 2 ** 16 + word[..., 3] * 2 ** 24
    n = torch.stack([(word // 16 ** (j // 2 + 4 * (j % 2))) % 16 for j in range(8)], dim=-1).flatten(-2)
    b = s[x + "_scale"][l, :, :, :s["cache"]].double()
    scale = (1 + torch.remainder(b, 8) / 8) * torch.exp2(torch.floor(b / 8) - BIAS)
    return (n - 8).double() * scale.repeat_interleave(GROUP, dim=-1)


def _rounded64(x):
    """The values that the 4-bit rows hold for x."""
    g = x.double().unflatten(-1, (-1, GROUP))
    amax = g.abs().amax(dim=-1, keepdim=True)
    m, e = torch.frexp(amax / torch.full_like(amax, 7))               # m in [0.5, 1)
    scale = torch.ldexp(torch.round(m * 16) / 16, e).clamp(2.0 ** -BIAS, 3840.0)
    return (torch.round(g / scale) * scale).flatten(-2)


def exact(case, seed):
    if case["kind"] == "evict":
        return None                                                   # nothing is computed but places
    s = prepare(case, seed)
    B, nl, Hq, Hkv, D = case["batch"], case["layers"], case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    if case["kind"] == "commit":
        res = {}
        for x in ("k", "v"):
            res[x] = torch.zeros(nl, B, Hkv, case["rows"], D, dtype=torch.float64, device=DEVICE)
            for b, n in enumerate(_n_rows(case)):
                take = s["src_idx"][b, :n].long() if case["scatter"] else torch.arange(n, device=DEVICE)
                res[x][:, b, :, :n] = _rounded64(s[x + "_new"][:, b][:, :, take])
        return res
    lc, lq = _lengths(case)
    L, g = case["block"], Hq // Hkv
    out = torch.zeros(nl, B, Hq, L, D, dtype=torch.float64, device=DEVICE)
    lse = torch.full((nl, B, Hq, L), -math.inf, dtype=torch.float64, device=DEVICE)
    weight = s["collected"].double() if case["kind"] == "weight" else None
    for l in range(nl):
        k, v = _values64(s, "k", l), _values64(s, "v", l) if case["kind"] == "attn" else None
        for b in range(B):
            c, n = lc[b], lq[b]
            q = s["q"][l, b, :, :n].double().unflatten(0, (Hkv, g)).flatten(1, 2)             # [Hkv, g * n, D]
            if weight is not None:
                z = q @ k[b, :, :c].transpose(1, 2) / math.sqrt(D)
                z -= s["lse"][l, b, :, :n].double().reshape(Hkv, g * n, 1)
                weight[l, b, :, :c] = DECAY * weight[l, b, :, :c] + z.exp().sum(dim=1)
                continue
            z = q @ torch.cat([k[b, :, :c], s["k_new"][l, b, :, :n].double()], dim=1).transpose(1, 2) / math.sqrt(D)
            total = torch.logsumexp(z, dim=-1)
            lse[l, b, :, :n] = total.reshape(Hq, n)
            o = (z - total[..., None]).exp() @ torch.cat([v[b, :, :c], s["v_new"][l, b, :, :n].double()], dim=1)
            out[l, b, :, :n] = o.reshape(Hq, n, D)
    return {"weight": weight} if weight is not None else {"out": out, "lse": lse}
