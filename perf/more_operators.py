"""Cases for a paged key / value cache held in 8 bits: keys and values quantised as they are written, read
back, and attended to.

An element is an e4m3 number, with a scale for each block of 16 tokens of a page and each key / value head:
the smallest power of two that brings the block's largest magnitude to 448 or less, held as its exponent in
8 bits (e8m0). A block grows with its tokens: its scale is that of all tokens written to it so far, and what
it held is rounded anew when the scale rises. Writing a block's first token begins it anew.

kinds:
  write       queries rotated; keys rotated and quantised into the cache, values quantised into it; the
              requests' new tokens follow what their last blocks hold already
  read        tokens at given slots, read back in 16 bits
  attention   attention of every request's new tokens over its pages, causal; a group of query heads
              shares a key / value head

A case's lengths follow from its numbers alone (`mix` seeds them), so that its work is known without a
GPU; values, page order and slots follow from the seed. Caches hold NaN, elements and scales alike, outside
the tokens that requests own, as memory that nobody has written may.
"""
import math
import random

import torch

own = False
DEV = "cuda"
BLOCK = 16
TOP = 448.0  # the largest e4m3 number
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _case(name, kind, **more):
    return dict({"name": name, "kind": kind}, **more)


def listed():
    return [
        # one decode step of 8 sequences through a 4096-wide layer: one token each, somewhere in a block
        _case("write_decode_T8", "write", B=8, decodes=8, new_lo=1, new_hi=1, old_lo=100, old_hi=4000, heads=32, kv_heads=32, d=128, rot=128, layout="half", page=16, dtype="bf16", scaled=False, mix=1),
        # a decode step of 200 sequences of a wider model, shared key / value heads
        _case("write_decode_T200", "write", B=200, decodes=200, new_lo=1, new_hi=1, old_lo=100, old_hi=30000, heads=64, kv_heads=8, d=128, rot=128, layout="half", page=64, dtype="bf16", scaled=True, mix=2),
        # a chunk of 8192 tokens late in a long context, beginning inside a block
        _case("write_chunk_T8192", "write", B=1, decodes=0, new_lo=8192, new_hi=8192, old_lo=100007, old_hi=100007, heads=64, kv_heads=8, d=128, rot=128, layout="half", page=64, dtype="bf16", scaled=True, mix=3),
        # part of each head rotated, neighbouring pairs, ragged requests, fp16
        _case("write_part_d64", "write", B=9, decodes=3, new_lo=20, new_hi=301, old_lo=0, old_hi=5000, heads=12, kv_heads=4, d=64, rot=32, layout="interleaved", page=16, dtype="fp16", scaled=False, mix=4),
        # one short request handed on
        _case("read_T301", "read", T=301, kv_heads=8, d=128, page=16, dtype="bf16"),
        # a long context read back
        _case("read_T50001", "read", T=50001, kv_heads=8, d=128, page=64, dtype="bf16"),
        # one short sequence, one new token, 32 heads: latency
        _case("attn_decode_B1", "attention", B=1, decodes=1, new_lo=1, new_hi=1, old_lo=350, old_hi=350, heads=32, kv_heads=32, d=128, page=16, dtype="bf16", mix=5),
        # 64 sequences of very unlike lengths, shared key / value heads
        _case("attn_decode_gqa_B64", "attention", B=64, decodes=64, new_lo=1, new_hi=1, old_lo=500, old_hi=20000, heads=64, kv_heads=8, d=128, page=64, dtype="bf16", mix=6),
        # one very long sequence
        _case("attn_decode_ctx100k", "attention", B=1, decodes=1, new_lo=1, new_hi=1, old_lo=100000, old_hi=100000, heads=64, kv_heads=8, d=128, page=64, dtype="bf16", mix=7),
        # a new prompt through a 4096-wide layer
        _case("attn_prompt_T1900", "attention", B=1, decodes=0, new_lo=1900, new_hi=1900, old_lo=0, old_hi=0, heads=32, kv_heads=32, d=128, page=16, dtype="bf16", mix=8),
        # a chunk late in a long context, shared key / value heads
        _case("attn_chunk_T2048_ctx30k", "attention", B=1, decodes=0, new_lo=2048, new_hi=2048, old_lo=30001, old_hi=30001, heads=64, kv_heads=8, d=128, page=64, dtype="bf16", mix=9),
        # sequences in decode beside two chunks, smaller heads, fp16
        _case("attn_mixed_B18_d64", "attention", B=18, decodes=16, new_lo=150, new_hi=601, old_lo=30, old_hi=2000, heads=16, kv_heads=4, d=64, page=16, dtype="fp16", mix=10),
    ]


# ---- draws ---------------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "write", "read", "attention", "attention", "attention", "attention"])
    mix, dtype, d = rng.randrange(1 << 20), rng.choice(["bf16", "bf16", "fp16"]), rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    kv = rng.choice([1, 2, 4, 8, 8, 32])
    heads = kv * rng.choice([1, 2, 3, 4, 7, 8] if kv <= 8 else [1, 2])
    if kind == "read":
        return {"kind": kind, "T": _log(rng, 1, 50000 if kv <= 8 else 10000), "kv_heads": kv, "d": d, "page": page, "dtype": dtype}
    shape = {"heads": heads, "kv_heads": kv, "d": d, "page": page, "dtype": dtype, "mix": mix}
    if kind == "write":
        shape.update(rot=rng.choice([d, d, d // 2]), layout=rng.choice(["half", "interleaved"]), scaled=rng.random() < 0.5)
        form = rng.choice(["decode", "chunk", "mixed"])
        if form == "decode":
            B = _log(rng, 1, 300)
            return dict({"kind": kind, "B": B, "decodes": B, "new_lo": 1, "new_hi": 1, "old_lo": 0, "old_hi": _log(rng, 1, 100000)}, **shape)
        if form == "chunk":
            new, old = _log(rng, 1, 8192 if kv <= 8 else 4096), rng.choice([0, 1, 1]) * _log(rng, 1, 100000)
            return dict({"kind": kind, "B": 1, "decodes": 0, "new_lo": new, "new_hi": new, "old_lo": old, "old_hi": old}, **shape)
        B, new = rng.randint(2, 30), _log(rng, 2, 250)
        return dict({"kind": kind, "B": B, "decodes": rng.randint(0, B - 1), "new_lo": 1 + new // 4, "new_hi": new, "old_lo": 0, "old_hi": _log(rng, 50, 20000)}, **shape)
    form = rng.choice(["decode", "few", "chunk", "mixed"])
    if form == "decode":  # one new token each
        B = _log(rng, 1, 64)
        hi = _log(rng, 64, 6000 if kv > 8 else 20000 if B > 8 else 100000)
        return dict({"kind": kind, "B": B, "decodes": B, "new_lo": 1, "new_hi": 1, "old_lo": rng.choice([0, hi // 40]), "old_hi": hi}, **shape)
    if form == "few":  # a handful of new tokens each
        B, hi = _log(rng, 1, 32), _log(rng, 64, 8000)
        return dict({"kind": kind, "B": B, "decodes": 0, "new_lo": 1, "new_hi": rng.randint(2, 17), "old_lo": rng.choice([0, hi // 8]), "old_hi": hi}, **shape)
    if form == "chunk":
        new, old = _log(rng, 17, 2048), rng.choice([0, 1, 1]) * _log(rng, 1, 30000)
        return dict({"kind": kind, "B": 1, "decodes": 0, "new_lo": new, "new_hi": new, "old_lo": old, "old_hi": old}, **shape)
    B, new = rng.randint(2, 16), _log(rng, 17, 500)
    return dict({"kind": kind, "B": B, "decodes": rng.randint(0, B - 1), "new_lo": 1 + new // 4, "new_hi": new, "old_lo": 0, "old_hi": _log(rng, 50, 2000)}, **shape)


# ---- lengths and inputs ----------------------------------------------------------------------------
def _spread(rng, lo, hi):
    return lo + int((hi - lo + 1) ** rng.random()) - 1 if hi > lo else lo


def _lengths(case):
    """(new, cached) tokens of each request."""
    rng = random.Random(case["mix"])
    new = [1 if b < case["decodes"] else _spread(rng, case["new_lo"], case["new_hi"]) for b in range(case["B"])]
    old = [_spread(rng, case["old_lo"], case["old_hi"]) for _ in new]
    order = list(range(case["B"]))
    rng.shuffle(order)
    return [new[b] for b in order], [old[b] for b in order]


def _dtype(case):
    return torch.float16 if case["dtype"] == "fp16" else torch.bfloat16


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _randn(gen, *shape, dtype=None, scale=1.0):
    x = torch.randn(shape, device=DEV, generator=gen)
    return x if dtype is None else (x * scale).to(dtype)


def _frequencies(rot, scaled):
    """Turns per position, times 2^64: base 10000; scaled: base 500000 with slow pairs eight times slower,
    those that turn 1 to 4 times in 8192 positions blended."""
    out = []
    for i in range(rot // 2):
        f = (500000.0 if scaled else 10000.0) ** (-2.0 * i / rot) / (2.0 * math.pi)
        if scaled:
            keep = min(1.0, max(0.0, (8192.0 * f - 1.0) / 3.0))
            f = f * (keep + (1.0 - keep) / 8.0)
        out.append(int(f * 2.0 ** 64))
    return torch.tensor(out, dtype=torch.int64, device=DEV)


def _pow2(n):
    """2^n in fp32, exactly, for whole n from -126 to 127."""
    return ((n.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent(a):
    """The exponent of the smallest power of two that brings magnitudes a to 448 = 0.875 2^9 or less."""
    m, e = torch.frexp(a)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(a > 0, e, -126).clamp(-126, 120)


def _values(gen, shape, spread):
    """Magnitudes that differ from token to token, and for some columns of keys."""
    x = _randn(gen, *shape) * torch.exp(0.4 * _randn(gen, *shape[:-2], 1, 1))
    return x * torch.where(torch.rand(shape[-1], device=DEV, generator=gen) < 0.03, spread, 1.0)


def _quantised(x, owned):
    """Cache and scales of values x (pages x page_size x heads x d) where requests own tokens, NaN elsewhere."""
    pages, P, Hk, d = x.shape
    x = torch.where(owned, x, 0.0).view(pages, P // BLOCK, BLOCK, Hk, d)
    e = _exponent(x.abs().amax((2, 4)))
    q = (x * _pow2(-e)[:, :, None, :, None]).to(E4M3).view(torch.uint8).view(pages, P, Hk, d)
    some = owned.view(pages, P // BLOCK, BLOCK, 1).any(2)
    scale = torch.where(some, e + 127, 255).to(torch.uint8)
    return torch.where(owned, q, 127).view(E4M3), scale.contiguous().view(E8M0)


def _paged(gen, case, new, old, extra):
    """Tables over shuffled pages for requests of old + new tokens, and a cache with `extra` of the new ones filled in
    as well as the old ones."""
    P, Hk, d = case["page"], case["kv_heads"], case["d"]
    want = [-(-(a + b) // P) for a, b in zip(new, old)]
    pages = sum(want) + 3
    order = torch.randperm(pages, device=DEV, generator=gen).to(torch.int32)
    first = _i32([sum(want[:b]) for b in range(len(want))])
    cols = torch.arange(max(want), dtype=torch.int32, device=DEV)
    inside = cols[None] < _i32(want)[:, None]
    at = torch.where(inside, first[:, None] + cols[None], 0)
    table = torch.where(inside, order[at.long()], -1).contiguous()
    held = _i32([b + (a if extra else 0) for a, b in zip(new, old)])
    owned = torch.zeros(pages * P + P, dtype=torch.bool, device=DEV)  # the last P: for places outside any request
    tok = torch.arange(max(want) * P, device=DEV)
    page = table.long()[:, tok // P]
    owned[torch.where(tok[None] < held[:, None], page * P + tok % P, pages * P)] = True
    owned = owned[:pages * P].view(pages, P, 1, 1)
    k, ks = _quantised(_values(gen, (pages, P, Hk, d), 4.0) * 1.5, owned)
    v, vs = _quantised(_values(gen, (pages, P, Hk, d), 1.0), owned)
    return {"k_cache": k, "v_cache": v, "k_scale": ks, "v_scale": vs, "table": table}


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    kind = case["kind"]
    state = {"case": case}
    dt, P, Hk, d = _dtype(case), case["page"], case["kv_heads"], case["d"]
    if kind == "read":
        T = case["T"]
        state.update(_paged(gen, case, [T], [0], True))
        t = torch.arange(T, device=DEV)
        state["slots"] = state["table"][0].long()[t // P] * P + t % P
        state["K"], state["V"] = (torch.empty((T, Hk, d), dtype=dt, device=DEV) for _ in range(2))
        return state
    new, old = _lengths(case)
    H, T = case["heads"], sum(new)
    start = [sum(new[:b]) for b in range(len(new) + 1)]
    if kind == "write":  # of the cached tokens only those of the page that is written further are there
        state.update(_paged(gen, case, new, [o % P for o in old], False))
        qkv = _randn(gen, T, H + 2 * Hk, d)  # one projection's output, queries, keys and values side by side
        qkv[:, H:] = _values(gen, (T, 2 * Hk, d), 2.0) * 1.3
        qkv = qkv.to(dt)
        state["Q"], state["K"], state["V"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        state["Qr"] = torch.empty((T, H, d), dtype=dt, device=DEV)
        state["freq"] = _frequencies(case["rot"], case["scaled"])
        t = torch.arange(T, device=DEV)
        b = torch.searchsorted(torch.tensor(start[1:], device=DEV), t, right=True)
        i = t - torch.tensor(start, device=DEV)[b]
        state["positions"] = (torch.tensor(old, device=DEV)[b] + i).to(torch.int32)
        at = torch.tensor([o % P for o in old], device=DEV)[b] + i
        state["slots"] = state["table"].long()[b, at // P] * P + at % P
        return state
    state.update(_paged(gen, case, new, old, True))
    state["q_start"], state["kv_len"] = _i32(start), _i32([a + b for a, b in zip(new, old)])
    state["Q"] = _randn(gen, T, H, d, dtype=dt, scale=1.3)
    state["O"] = torch.empty_like(state["Q"])
    state["max_q"] = max(new)
    state["scale"] = d ** -0.5
    return state


# ---- the plain forms: 32 bits, rounded once ----------------------------------------------------------
def _plain_rotate(x, positions, freq, layout):
    phase = (positions.long()[:, None] * freq[None]) >> 32  # the product wraps at one turn
    angle = (phase.float() * (2.0 * math.pi / 2.0 ** 32))[:, None]
    c, sn = torch.cos(angle), torch.sin(angle)
    n = freq.numel()
    y = x.float().clone()
    one, two = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = y[..., one].clone(), y[..., two].clone()
    y[..., one], y[..., two] = a * c - b * sn, b * c + a * sn
    return y


def _plain_store(cache, scale, x, slots):
    """x (T x heads x d, fp32) quantised into the cache at its slots."""
    Hk, d = cache.shape[2:]
    held = scale.view(torch.uint8).view(-1, Hk)
    blk, off = slots // BLOCK, slots % BLOCK
    most = torch.zeros(held.shape, device=x.device).index_reduce_(0, blk, x.abs().amax(-1), "amax")
    first = torch.full((held.shape[0],), BLOCK, device=x.device).index_reduce_(0, blk, off, "amin")[:, None]
    was, e = held.int() - 127, _exponent(most)
    grown = first.gt(0) & first.lt(BLOCK)  # blocks that held tokens before
    e = torch.where(grown, torch.maximum(was, e), e)
    data = cache.view(-1, BLOCK, Hk, d).float()
    data = (data * _pow2(torch.where(grown, (was - e).clamp(min=-126), 0))[:, None, :, None]).view(-1, Hk, d)
    data[slots] = x * _pow2(-e)[blk][..., None]
    cache.copy_(data.to(E4M3).view(cache.shape))
    held.copy_(torch.where(first < BLOCK, e + 127, held.int()))


def _plain_values(cache, scale):
    """fp32 values of a cache (or of pages of it)."""
    n = scale.view(torch.uint8).int() - 127
    s = torch.where(n < 128, _pow2(n.clamp(-126, 127)), math.nan)
    return cache.float() * s.repeat_interleave(BLOCK, -2)[..., None]


def _plain_pages(cache, scale, pages):
    """fp32 values of the tokens of some pages (B x columns), B x tokens x heads x d."""
    x = _plain_values(cache.view(torch.uint8)[pages].view(E4M3), scale.view(torch.uint8)[pages].view(E8M0))
    return x.flatten(1, 2)


def _plain_attention(s):
    c = s["case"]
    H, Hk, d, P = c["heads"], c["kv_heads"], c["d"], c["page"]
    Q, table, start, kv_len = s["Q"], s["table"], s["q_start"].long(), s["kv_len"].long()
    B, T, mq, L = kv_len.numel(), Q.shape[0], s["max_q"], table.shape[1] * P
    i, j = torch.arange(mq, device=Q.device), torch.arange(L, device=Q.device)
    q = Q[(start[:B, None] + i[None]).clamp(max=T - 1)].float().view(B, mq, Hk, H // Hk, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, -1, d)
    pages = table.long().clamp(min=0)
    gone = (j[None] >= kv_len[:, None])[..., None, None]
    k = _plain_pages(s["k_cache"], s["k_scale"], pages).masked_fill_(gone, 0.0).transpose(1, 2)
    v = _plain_pages(s["v_cache"], s["v_scale"], pages).masked_fill_(gone, 0.0).transpose(1, 2)
    a = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).view(B, Hk, H // Hk, mq, L)
    last = (kv_len - (start[1:] - start[:-1]))[:, None] + i[None]  # the last key that a row sees
    a.masked_fill_((j > last[..., None])[:, None, None], -math.inf)
    a.sub_(a.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = a.sum(-1, keepdim=True)
    o = torch.matmul(a.view(B, Hk, -1, L), v).view(B, Hk, H // Hk, mq, d) / total.clamp(min=1e-37)
    t = torch.arange(T, device=Q.device)
    b = torch.searchsorted(start[1:].contiguous(), t, right=True)
    return o.permute(0, 3, 1, 2, 4)[b, t - start[b]].reshape(T, H, d).to(Q.dtype)


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "write":
        _plain_store(s["k_cache"], s["k_scale"], _plain_rotate(s["K"], s["positions"], s["freq"], c["layout"]), s["slots"])
        _plain_store(s["v_cache"], s["v_scale"], s["V"].float(), s["slots"])
        Qr = _plain_rotate(s["Q"], s["positions"], s["freq"], c["layout"]).to(s["Q"].dtype)
        return {"Qr": Qr, "k_cache": s["k_cache"], "v_cache": s["v_cache"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if c["kind"] == "read":
        at = (s["slots"] // c["page"], s["slots"] % c["page"])
        return {n: _plain_values(s[m + "_cache"], s[m + "_scale"])[at].to(s[n].dtype) for n, m in (("K", "k"), ("V", "v"))}
    return _plain_attention(s)


# ---- the framework's operators -----------------------------------------------------------------------
def _run_own(s):
    from paper_2501_19090_gb300 import pifa as P

    c = s["case"]
    cache = (s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    if c["kind"] == "write":
        layout = P.PIFA_ROPE_HALF if c["layout"] == "half" else P.PIFA_ROPE_INTERLEAVED
        Qr = P.pifa_rope_cache_q8(s["Q"], s["K"], s["V"], s["positions"], s["slots"], s["freq"], *cache, layout, Qr=s["Qr"])
        return {"Qr": Qr, "k_cache": s["k_cache"], "v_cache": s["v_cache"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if c["kind"] == "read":
        K, V = P.pifa_cache_read_q8(*cache, s["slots"], K=s["K"], V=s["V"])
        return {"K": K, "V": V}
    return P.pifa_paged_attention_q8(s["Q"], *cache, s["table"], s["q_start"], s["kv_len"], s["max_q"], scale=s["scale"], O=s["O"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------
def work(case):
    Hk, d, kind = case["kv_heads"], case["d"], case["kind"]
    if kind == "read":  # elements in 8 bits in, in 16 out; the blocks' scales; the slots
        T = case["T"]
        return {"bytes": 6 * T * Hk * d + 2 * -(-T // BLOCK) * Hk + 8 * T, "flops": 2 * T * Hk * d}
    new, old = _lengths(case)
    H, T = case["heads"], sum(new)
    if kind == "write":
        # queries in and out, keys and values in and, in 8 bits, out; scales of the touched blocks out, and in where
        # they held tokens; positions, slots, frequencies
        touched = sum(-(-(a + b) // BLOCK) - b // BLOCK for a, b in zip(new, old))
        held = sum(b % BLOCK > 0 for b in old)
        return {"bytes": 4 * T * H * d + 6 * T * Hk * d + 2 * (touched + held) * Hk + 12 * T + 4 * case["rot"],
                "flops": 3 * T * (H + Hk) * case["rot"] + 4 * T * Hk * d}
    pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(new, old))
    kv = T + sum(old)
    blocks = sum(-(-(a + b) // BLOCK) for a, b in zip(new, old))
    return {"bytes": 4 * T * H * d + 2 * kv * Hk * d + 2 * blocks * Hk + 4 * kv // case["page"] + 8 * case["B"], "flops": 4 * d * H * pairs}


# ---- the same in 64 bits ---------------------------------------------------------------------------------
def _exact_rotate(x, s):
    """As complex numbers."""
    turns = s["positions"].double()[:, None] * (s["freq"].double() * 2.0 ** -64)
    turn = torch.polar(torch.ones_like(turns), 2.0 * math.pi * (turns - turns.round()))[:, None]
    n = s["freq"].numel()
    head = x[..., :2 * n].double()
    pairs = head.unflatten(-1, (2, n)).transpose(-1, -2) if s["case"]["layout"] == "half" else head.unflatten(-1, (n, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    z = z.transpose(-1, -2) if s["case"]["layout"] == "half" else z
    return torch.cat([z.flatten(-2), x[..., 2 * n:].double()], -1)


def _exact_store(cache, scale, x, slots):
    """Block by block, in the order of the tokens: elements before they are rounded, in units of the scales."""
    Hk, d = cache.shape[2:]
    data, held = cache.double().view(-1, BLOCK, Hk, d), scale.double().view(-1, Hk)
    at = slots.tolist()
    begin = 0
    while begin < len(at):
        end = begin + 1
        while end < len(at) and at[end] // BLOCK == at[begin] // BLOCK:
            end += 1
        block, offs = at[begin] // BLOCK, [t % BLOCK for t in at[begin:end]]
        new = x[begin:end]
        most = new.abs().amax((0, 2))
        s = torch.exp2(torch.ceil(torch.log2(most / TOP)))
        s = torch.where(most <= TOP * s / 2, s / 2, s)  # a logarithm next to a whole number may be off by its last bit
        if min(offs) > 0:
            s = torch.maximum(s, held[block])
            data[block] *= (held[block] / s)[None, :, None]
        data[block, offs] = new / s[None, :, None]
        held[block] = s
        begin = end
    return data.view(cache.shape), held.view(scale.shape)


def _exact_attention(s):
    """Request by request and head by head."""
    c = s["case"]
    G = c["heads"] // c["kv_heads"]
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEV)
    start, lens = s["q_start"].tolist(), s["kv_len"].tolist()

    def values(which, pages, n):
        x, f = (s[which + t].view(torch.uint8)[pages] for t in ("_cache", "_scale"))
        x, f = x.view(E4M3).double().flatten(0, 1)[:n], f.view(E8M0).double().flatten(0, 1)
        return x * f[torch.arange(n, device=DEV) // BLOCK][..., None]

    for b, n in enumerate(lens):
        pages = s["table"][b, : -(-n // c["page"])].long()
        k, v = values("k", pages, n), values("v", pages, n)
        q = s["Q"][start[b]:start[b + 1]].double()
        sees = torch.ones((q.shape[0], n), dtype=torch.bool, device=DEV).tril(n - q.shape[0])
        for h in range(c["heads"]):
            a = (q[:, h] @ k[:, h // G].t() * s["scale"]).masked_fill(~sees, -math.inf)
            out[start[b]:start[b + 1], h] = torch.softmax(a, -1) @ v[:, h // G]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "write":
        k, ks = _exact_store(s["k_cache"], s["k_scale"], _exact_rotate(s["K"], s), s["slots"])
        v, vs = _exact_store(s["v_cache"], s["v_scale"], s["V"].double(), s["slots"])
        return {"Qr": _exact_rotate(s["Q"], s), "k_cache": k, "v_cache": v, "k_scale": ks, "v_scale": vs}
    if case["kind"] == "read":
        P, at = case["page"], s["slots"].tolist()
        out = {}
        for name, which in (("K", "k"), ("V", "v")):
            x = s[which + "_cache"].view(torch.uint8).view(-1, *s[which + "_cache"].shape[2:])[at].view(E4M3).double()
            f = s[which + "_scale"].view(torch.uint8).view(-1, case["kv_heads"])[[t // P * (P // BLOCK) + t % P // BLOCK for t in at]]
            out[name] = x * f.view(E8M0).double()[..., None]
        return out
    return _exact_attention(s)
