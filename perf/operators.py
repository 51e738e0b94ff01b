"""Cases for the operators between a layer's projections: page tables, rotary positions and attention
over a paged cache.

kinds:
  tables      page tables, slot map and positions of one step, from the requests' lengths
  rope        rotary positions of one projection's output and their gradient, as a training step has them
  rope_cache  queries rotated, keys rotated into the paged cache, values copied into it
  attention   attention of every request's new tokens over its pages, causal; a group of query heads
              shares a key/value head

A case's lengths follow from its numbers alone (`mix` seeds them), so that its work is known without a
GPU; values, page order and free lists follow from the seed. Caches hold NaN outside the tokens that
requests own, as memory that nobody has written may. Frequencies are turns per position in units of
2^-64 turn, so that a position's phase is an integer product modulo one turn.
"""
import math
import random

import torch

own = False
DEV = "cuda"


def _case(name, kind, **more):
    return dict({"name": name, "kind": kind}, **more)


def listed():
    return [
        # a decode step of 64 sequences: a new page now and then
        _case("tables_decode_B64", "tables", B=64, decodes=64, new_lo=1, new_hi=1, old_lo=100, old_hi=8000, page=16, mix=1),
        # a large step: 500 sequences decode, 20 bring chunks; padded to the step's token capacity
        _case("tables_step_B520", "tables", B=520, decodes=500, new_lo=100, new_hi=1500, old_lo=1, old_hi=30000, page=64, mix=2),
        # one step of 8 sequences through a 4096-wide layer: 32 heads of 128
        _case("rope_cache_T8", "rope_cache", T=8, heads=32, kv_heads=32, d=128, rot=128, layout="half", page=16, dtype="bf16", far=4000, scaled=False),
        # a chunk through an 8192-wide layer with shared key/value heads, at positions of a long context
        _case("rope_cache_T8192", "rope_cache", T=8192, heads=64, kv_heads=8, d=128, rot=128, layout="half", page=64, dtype="bf16", far=120000, scaled=True),
        # a training step's queries, forward and gradient
        _case("rope_train_T2048", "rope", T=2048, heads=32, d=128, rot=128, layout="half", dtype="bf16", far=1, scaled=False),
        # part of each head rotated, neighbouring pairs, an odd token count, fp16
        _case("rope_train_part_T1001", "rope", T=1001, heads=12, d=64, rot=32, layout="interleaved", dtype="fp16", far=5000, scaled=False),
        # one short sequence, one new token, 32 heads: latency
        _case("attn_decode_B1", "attention", B=1, decodes=1, new_lo=1, new_hi=1, old_lo=300, old_hi=300, heads=32, kv_heads=32, d=128, page=16, dtype="bf16", mix=3),
        # a batch of 8 sequences through a 4096-wide layer
        _case("attn_decode_B8", "attention", B=8, decodes=8, new_lo=1, new_hi=1, old_lo=1000, old_hi=4095, heads=32, kv_heads=32, d=128, page=16, dtype="bf16", mix=4),
        # 64 sequences of very unlike lengths, shared key/value heads
        _case("attn_decode_gqa_B64", "attention", B=64, decodes=64, new_lo=1, new_hi=1, old_lo=400, old_hi=16000, heads=64, kv_heads=8, d=128, page=64, dtype="bf16", mix=5),
        # a new prompt through a 4096-wide layer
        _case("attn_prompt_T2048", "attention", B=1, decodes=0, new_lo=2048, new_hi=2048, old_lo=0, old_hi=0, heads=32, kv_heads=32, d=128, page=16, dtype="bf16", mix=6),
        # a chunk late in a long context, shared key/value heads
        _case("attn_chunk_T2048_ctx30k", "attention", B=1, decodes=0, new_lo=2048, new_hi=2048, old_lo=30000, old_hi=30000, heads=64, kv_heads=8, d=128, page=64, dtype="bf16", mix=7),
        # sequences in decode beside two chunks, smaller heads, fp16
        _case("attn_mixed_B18_d64", "attention", B=18, decodes=16, new_lo=150, new_hi=601, old_lo=30, old_hi=2000, heads=16, kv_heads=4, d=64, page=16, dtype="fp16", mix=8),
    ]


# ---- draws ---------------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tables", "rope", "rope_cache", "attention", "attention", "attention", "attention"])
    mix, dtype, d = rng.randrange(1 << 20), rng.choice(["bf16", "bf16", "fp16"]), rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    if kind == "tables":
        B = _log(rng, 1, 520)
        return {"kind": kind, "B": B, "decodes": int(B * rng.choice([1.0, 0.95, 0.5])), "new_lo": 1,
                "new_hi": _log(rng, 1, 1500), "old_lo": 1, "old_hi": _log(rng, 100, 30000), "page": page, "mix": mix}
    rot = rng.choice([d, d, d // 2])
    layout, scaled = rng.choice(["half", "interleaved"]), rng.random() < 0.5
    if kind == "rope":
        return {"kind": kind, "T": _log(rng, 1, 4096), "heads": rng.randint(1, 64), "d": d, "rot": rot, "layout": layout,
                "dtype": dtype, "far": _log(rng, 1, 120000), "scaled": scaled}
    kv = rng.choice([1, 2, 4, 8, 8, 32])
    heads = kv * rng.choice([1, 2, 3, 4, 7, 8] if kv <= 8 else [1, 2])
    if kind == "rope_cache":
        return {"kind": kind, "T": _log(rng, 1, 8192), "heads": heads, "kv_heads": kv, "d": d, "rot": rot,
                "layout": layout, "page": page, "dtype": dtype, "far": _log(rng, 1, 120000), "scaled": scaled}
    shape = {"heads": heads, "kv_heads": kv, "d": d, "page": page, "dtype": dtype, "mix": mix}
    form = rng.choice(["decode", "few", "chunk", "mixed"])
    if form == "decode":  # one new token each
        B, hi = _log(rng, 1, 64), _log(rng, 64, 16000)
        return dict({"kind": kind, "B": B, "decodes": B, "new_lo": 1, "new_hi": 1, "old_lo": rng.choice([0, hi // 40]), "old_hi": hi}, **shape)
    if form == "few":  # a handful of new tokens each
        B, hi = _log(rng, 1, 32), _log(rng, 64, 8000)
        return dict({"kind": kind, "B": B, "decodes": 0, "new_lo": 1, "new_hi": rng.randint(2, 17), "old_lo": rng.choice([0, hi // 8]), "old_hi": hi}, **shape)
    if form == "chunk":
        new = _log(rng, 17, 2048)
        old = rng.choice([0, 1, 1]) * _log(rng, 1, 30000)
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


def _paged(gen, case):
    """Lengths, tables over shuffled pages, and a cache filled where requests own tokens."""
    new, old = _lengths(case)
    P, Hk, d = case["page"], case["kv_heads"], case["d"]
    want = [-(-(a + b) // P) for a, b in zip(new, old)]
    pages = sum(want) + 3
    order = torch.randperm(pages, device=DEV, generator=gen).to(torch.int32)
    first = _i32([sum(want[:b]) for b in range(len(want))])
    cols = torch.arange(max(want), dtype=torch.int32, device=DEV)
    inside = cols[None] < _i32(want)[:, None]
    at = torch.where(inside, first[:, None] + cols[None], 0)
    table = torch.where(inside, order[at.long()], -1).contiguous()
    kv_len = _i32([a + b for a, b in zip(new, old)])
    owned = torch.zeros(pages * P + P, dtype=torch.bool, device=DEV)  # the last P: for places outside any request
    tok = torch.arange(max(want) * P, device=DEV)
    page = table.long()[:, tok // P]
    owned[torch.where(tok[None] < kv_len[:, None], page * P + tok % P, pages * P)] = True
    owned = owned[:pages * P].view(pages, P, 1, 1)
    k, v = (torch.where(owned, _randn(gen, pages, P, Hk, d, dtype=_dtype(case), scale=s), math.nan) for s in (1.5, 1.0))
    start = [sum(new[:b]) for b in range(len(new) + 1)]
    return {"k_cache": k, "v_cache": v, "table": table, "q_start": _i32(start), "kv_len": kv_len}, new


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    kind = case["kind"]
    state = {"case": case}
    if kind == "tables":
        new, old = _lengths(case)
        P = case["page"]
        have, want = [-(-a // P) for a in old], [-(-(a + b) // P) for a, b in zip(old, new)]
        pages = sum(want) + 9  # some free pages are left over, some entries of the list are already used
        order = torch.randperm(pages, device=DEV, generator=gen).to(torch.int32)
        cols = torch.arange(max(want) + 1, dtype=torch.int32, device=DEV)
        first = _i32([sum(have[:b]) for b in range(len(have))])
        inside = cols[None] < _i32(have)[:, None]
        table = torch.where(inside, order[torch.where(inside, first[:, None] + cols[None], 0).long()], -1).contiguous()
        tokens = -(-sum(new) // 8) * 8
        state.update(cached_len=_i32(old), new_len=_i32(new), table=table, free_pages=order, free_first=_i32([sum(have)]), tokens=tokens)
        state["out"] = (torch.empty(len(new) + 1, dtype=torch.int32, device=DEV), torch.empty(len(new), dtype=torch.int32, device=DEV),
                        torch.empty(tokens, dtype=torch.int32, device=DEV), torch.empty(tokens, dtype=torch.int64, device=DEV),
                        torch.empty(1, dtype=torch.int32, device=DEV))
        return state
    if kind in ("rope", "rope_cache"):
        T, H, d, dt = case["T"], case["heads"], case["d"], _dtype(case)
        state["freq"] = _frequencies(case["rot"], case["scaled"])
        state["positions"] = torch.randint(0, case["far"], (T,), device=DEV, generator=gen).to(torch.int32) if case["far"] > 1 \
            else torch.arange(T, dtype=torch.int32, device=DEV)
        if kind == "rope":
            state["X"], state["dY"] = _randn(gen, T, H, d, dtype=dt), _randn(gen, T, H, d, dtype=dt)
            state["Y"], state["dX"] = torch.empty_like(state["X"]), torch.empty_like(state["dY"])
            return state
        P, Hk = case["page"], case["kv_heads"]
        pages = -(-T // P) * 2 + 1
        qkv = _randn(gen, T, H + 2 * Hk, d, dtype=dt)  # one projection's output, queries, keys and values side by side
        state["Q"], state["K"], state["V"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        state["Qr"] = torch.empty((T, H, d), dtype=dt, device=DEV)
        runs = torch.randperm(pages, device=DEV, generator=gen)[: -(-T // P)]  # whole pages in order, as a chunk has them
        t = torch.arange(T, device=DEV)
        state["slots"] = runs[t // P] * P + t % P
        state["k_cache"], state["v_cache"] = (_randn(gen, pages, P, Hk, d, dtype=dt) for _ in range(2))
        return state
    paged, new = _paged(gen, case)
    state.update(paged)
    T, H, d = sum(new), case["heads"], case["d"]
    state["Q"] = _randn(gen, T, H, d, dtype=_dtype(case), scale=1.5)
    state["O"] = torch.empty_like(state["Q"])
    state["max_q"] = max(new)
    state["scale"] = d ** -0.5
    return state


# ---- the plain forms: 32 bits, rounded once ----------------------------------------------------------
def _plain_tables(s):
    P, T = s["case"]["page"], s["tokens"]
    old, new, table = s["cached_len"].long(), s["new_len"].long(), s["table"]
    have, want = (old + P - 1) // P, (old + new + P - 1) // P
    ends = torch.cumsum(want - have, 0)
    base = s["free_first"].long() + ends - (want - have) - have  # free-list entry of a request's page p: base + p
    zero = torch.zeros(1, dtype=torch.int64, device=table.device)
    start = torch.cat([zero, torch.cumsum(new, 0)])
    free = s["free_pages"]
    last = free.numel() - 1
    cols = torch.arange(table.shape[1], device=table.device)
    fresh = (cols[None] >= have[:, None]) & (cols[None] < want[:, None])
    table = torch.where(fresh, free[(base[:, None] + cols[None]).clamp(0, last)], table)
    t = torch.arange(T, device=table.device)
    b = torch.searchsorted(start[1:].contiguous(), t, right=True).clamp(max=new.numel() - 1)
    real = t < start[-1]
    pos = torch.where(real, old[b] + t - start[b], 0)
    slots = torch.where(real, table[b, pos // P].long() * P + pos % P, -1)
    return [table, start.int(), (old + new).int(), pos.int(), slots, (s["free_first"].long() + ends[-1:]).int()]


def _plain_rotate(x, positions, freq, layout, inverse=False):
    phase = (positions.long()[:, None] * freq[None]) >> 32  # the product wraps at one turn
    angle = (phase.float() * (2.0 * math.pi / 2.0 ** 32))[:, None]
    c, sn = torch.cos(angle), torch.sin(angle)
    if inverse:
        sn = -sn
    n = freq.numel()
    x32 = x.float()
    y = x32.clone()
    one, two = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    y[..., one] = x32[..., one] * c - x32[..., two] * sn
    y[..., two] = x32[..., two] * c + x32[..., one] * sn
    return y.to(x.dtype)


def _plain_attention(s):
    c = s["case"]
    H, Hk, d, P = c["heads"], c["kv_heads"], c["d"], c["page"]
    Q, table, start, kv_len = s["Q"], s["table"], s["q_start"].long(), s["kv_len"].long()
    B, T, mq, L = kv_len.numel(), Q.shape[0], s["max_q"], table.shape[1] * P
    i, j = torch.arange(mq, device=Q.device), torch.arange(L, device=Q.device)
    q = Q[(start[:B, None] + i[None]).clamp(max=T - 1)].float().view(B, mq, Hk, H // Hk, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, -1, d)
    pages = table.long().clamp(min=0)
    gone = (j[None] >= kv_len[:, None])[..., None, None]
    k, v = (x[pages].view(B, L, Hk, d).masked_fill(gone, 0.0).float().transpose(1, 2) for x in (s["k_cache"], s["v_cache"]))
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
    if c["kind"] == "tables":
        return _plain_tables(s)
    if c["kind"] == "rope":
        return {"Y": _plain_rotate(s["X"], s["positions"], s["freq"], c["layout"]),
                "dX": _plain_rotate(s["dY"], s["positions"], s["freq"], c["layout"], True)}
    if c["kind"] == "rope_cache":
        P = c["page"]
        at = (s["slots"] // P, s["slots"] % P)
        s["k_cache"][at] = _plain_rotate(s["K"], s["positions"], s["freq"], c["layout"])
        s["v_cache"][at] = s["V"]
        return {"Qr": _plain_rotate(s["Q"], s["positions"], s["freq"], c["layout"]), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    return _plain_attention(s)


# ---- the framework's operators -----------------------------------------------------------------------
def _run_own(s):
    from paper_2501_19090_gb300 import pifa as P

    c = s["case"]
    if c["kind"] == "tables":
        start, kv_len, pos, slots, nxt = P.pifa_page_tables(s["cached_len"], s["new_len"], c["page"], s["free_pages"], s["free_first"],
                                                            s["table"], s["tokens"], out=s["out"])
        return [s["table"], start, kv_len, pos, slots, nxt]
    if c["kind"] == "attention":
        return P.pifa_paged_attention(s["Q"], s["k_cache"], s["v_cache"], s["table"], s["q_start"], s["kv_len"], s["max_q"],
                                      scale=s["scale"], O=s["O"])
    layout = P.PIFA_ROPE_HALF if c["layout"] == "half" else P.PIFA_ROPE_INTERLEAVED
    if c["kind"] == "rope":
        return {"Y": P.pifa_rope(s["X"], s["positions"], s["freq"], layout, Y=s["Y"]),
                "dX": P.pifa_rope(s["dY"], s["positions"], s["freq"], layout, inverse=True, Y=s["dX"])}
    Qr = P.pifa_rope_cache(s["Q"], s["K"], s["V"], s["positions"], s["slots"], s["freq"], s["k_cache"], s["v_cache"], layout, Qr=s["Qr"])
    return {"Qr": Qr, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "tables":  # lengths in, sums out; per token its position and slot; per page its number in and, if new, out
        new, old = _lengths(case)
        P = case["page"]
        fresh = sum(-(-(a + b) // P) - -(-b // P) for a, b in zip(new, old))
        return {"bytes": 16 * case["B"] + 12 * sum(new) + 8 * fresh + 4 * sum(-(-a // P) for a in new), "flops": 0}
    if kind == "rope":  # forward and gradient: each element in and out
        n = case["T"] * case["heads"]
        return {"bytes": 2 * (4 * n * case["d"] + 4 * case["T"] + 4 * case["rot"]), "flops": 2 * 3 * n * case["rot"]}
    if kind == "rope_cache":
        T, H, Hk = case["T"], case["heads"], case["kv_heads"]
        return {"bytes": 4 * T * (H + 2 * Hk) * case["d"] + 12 * T + 4 * case["rot"], "flops": 3 * T * (H + Hk) * case["rot"]}
    new, old = _lengths(case)
    H, Hk, d = case["heads"], case["kv_heads"], case["d"]
    pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(new, old))
    kv = sum(new) + sum(old)
    return {"bytes": 4 * sum(new) * H * d + 4 * kv * Hk * d + 4 * kv // case["page"] + 8 * case["B"], "flops": 4 * d * H * pairs}


# ---- the same in 64 bits ---------------------------------------------------------------------------------
def _exact_tables(s):
    """Request by request, on the host."""
    P = s["case"]["page"]
    old, new, free = (s[k].tolist() for k in ("cached_len", "new_len", "free_pages"))
    table, nxt = s["table"].tolist(), int(s["free_first"])
    start, pos, slots = [0], [], []
    for b, (o, n) in enumerate(zip(old, new)):
        for t in range(o, o + n):
            if t % P == 0:
                table[b][t // P] = free[nxt]
                nxt += 1
            pos.append(t)
            slots.append(table[b][t // P] * P + t % P)
        start.append(start[-1] + n)
    pad = s["tokens"] - start[-1]
    return [_i32(table), _i32(start), _i32([a + b for a, b in zip(old, new)]), _i32(pos + [0] * pad),
            torch.tensor(slots + [-1] * pad, dtype=torch.int64, device=DEV), _i32([nxt])]


def _exact_rotate(x, s, sign=1.0):
    """As complex numbers."""
    turns = s["positions"].double()[:, None] * (s["freq"].double() * 2.0 ** -64)
    turn = torch.polar(torch.ones_like(turns), sign * 2.0 * math.pi * (turns - turns.round()))[:, None]
    n = s["freq"].numel()
    head = x[..., :2 * n].double()
    pairs = head.unflatten(-1, (2, n)).transpose(-1, -2) if s["case"]["layout"] == "half" else head.unflatten(-1, (n, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    z = z.transpose(-1, -2) if s["case"]["layout"] == "half" else z
    return torch.cat([z.flatten(-2), x[..., 2 * n:].double()], -1)


def _exact_attention(s):
    """Request by request and head by head."""
    c = s["case"]
    G = c["heads"] // c["kv_heads"]
    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEV)
    start, lens = s["q_start"].tolist(), s["kv_len"].tolist()
    for b, n in enumerate(lens):
        pages = s["table"][b, : -(-n // c["page"])].long()
        k, v = (x[pages].flatten(0, 1)[:n].double() for x in (s["k_cache"], s["v_cache"]))
        q = s["Q"][start[b]:start[b + 1]].double()
        sees = torch.ones((q.shape[0], n), dtype=torch.bool, device=DEV).tril(n - q.shape[0])
        for h in range(c["heads"]):
            a = (q[:, h] @ k[:, h // G].t() * s["scale"]).masked_fill(~sees, -math.inf)
            out[start[b]:start[b + 1], h] = torch.softmax(a, -1) @ v[:, h // G]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "tables":
        return _exact_tables(s)
    if case["kind"] == "rope":
        return {"Y": _exact_rotate(s["X"], s), "dX": _exact_rotate(s["dY"], s, -1.0)}
    if case["kind"] == "rope_cache":
        k, v, P = s["k_cache"].double(), s["v_cache"].double(), case["page"]
        k.view(-1, *k.shape[2:])[s["slots"]] = _exact_rotate(s["K"], s)
        v.view(-1, *v.shape[2:])[s["slots"]] = s["V"].double()
        return {"Qr": _exact_rotate(s["Q"], s), "k_cache": k, "v_cache": v}
    return _exact_attention(s)
