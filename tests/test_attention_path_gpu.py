"""GPU parity of what lies between the projections: page tables, rotary positions (with the cache write) and
attention over a paged cache, each against a plain implementation in 64 bits.

Page tables are whole numbers and have to be equal. Tolerances of the rest follow from the roundings
(u: 2^-8 for bf16, 2^-11 for fp16, the largest relative error of one rounding):
  rotary      one rounding of an fp32 result: u |y| + 1e-6 (|x| + |partner|) (fp32 sines, products, sum)
  attention   the weights are rounded once, the output once: u |o| + u sum_j p_j |v_j| (first order, 10% over
              for the rest), 2e-4 sum_j p_j |v_j| for fp32 scores, exponentials and sums, and for fp16
              2^-24 max |v| a key, for weights below the normal range
"""
import math
import random

import pytest
import torch

from paper_2501_19090_gb300 import pifa as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
DTYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    P.load()
    yield


@pytest.fixture(autouse=True)
def _clean_status():
    yield
    assert P.pifa_device_status() == P.PIFA_OK  # a test that expects an error has read it


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ---- page tables ---------------------------------------------------------------------------------------
def plain_tables(old, new, page, free, first, table, T):
    """Token by token."""
    start, pos, slots = [0], [], []
    for b, (o, n) in enumerate(zip(old, new)):
        for t in range(o, o + n):
            if t % page == 0:
                table[b][t // page] = free[first]
                first += 1
            pos.append(t)
            slots.append(table[b][t // page] * page + t % page)
        start.append(start[-1] + n)
    pad = T - len(pos)
    return table, start, [o + n for o, n in zip(old, new)], pos + [0] * pad, slots + [-1] * pad, first


def table_case(rng, B, page, most_old, most_new):
    old = [rng.choice([0, page, rng.randint(0, most_old)]) for _ in range(B)]
    new = [rng.choice([0, 1, 1, rng.randint(0, most_new)]) for _ in range(B)]
    have, want = [-(-o // page) for o in old], [-(-(o + n) // page) for o, n in zip(old, new)]
    order = list(range(sum(want) + 5))
    rng.shuffle(order)
    cols, at, table = max(want) + 2, 0, []
    for h in have:
        table.append(order[at:at + h] + [-7] * (cols - h))
        at += h
    return old, new, order, at, table


@pytest.mark.parametrize("B,page,most_old,most_new", [(1, 16, 0, 1), (1, 16, 40, 33), (3, 1, 9, 5), (7, 13, 100, 40),
                                                      (64, 16, 500, 1), (520, 64, 3000, 90), (1025, 32, 200, 3),
                                                      (4096, 16, 60, 20)])
def test_page_tables(B, page, most_old, most_new):
    rng = random.Random(B * 1000 + page)
    old, new, free, first, table = table_case(rng, B, page, most_old, most_new)
    T = sum(new) + rng.choice([0, 5])
    dev_table = i32(table)
    got = P.pifa_page_tables(i32(old), i32(new), page, i32(free), i32([first]), dev_table, T)
    want_table, start, kv, pos, slots, nxt = plain_tables(old, new, page, free, first, [list(r) for r in table], T)
    assert dev_table.tolist() == want_table
    assert [x.tolist() for x in got] == [start, kv, pos, slots, [nxt]]


def test_page_tables_steps_in_place():
    """A serving loop: lengths and the free list's head updated by the calls, in views of larger buffers."""
    rng = random.Random(4)
    B, page, cols = 37, 16, 40
    free = list(range(B * cols))
    rng.shuffle(free)
    lens, head = i32([0] * B), i32([0])
    table = torch.full((B, cols + 3), -1, dtype=torch.int32, device=DEV)[:, :cols]
    want, old, first = [[-1] * cols for _ in range(B)], [0] * B, 0
    for step in range(6):
        new = [rng.randint(0, 90) if step == 0 else rng.randint(0, 2) for _ in range(B)]
        T = 96 * B
        out = (torch.empty(B + 1, dtype=torch.int32, device=DEV), lens, torch.empty(T, dtype=torch.int32, device=DEV),
               torch.empty(T, dtype=torch.int64, device=DEV), head)
        P.pifa_page_tables(lens, i32(new), page, i32(free), head, table, T, out=out)
        want, start, old, pos, slots, first = plain_tables(old, new, page, free, first, want, T)
        assert table.tolist() == want and [x.tolist() for x in out] == [start, old, pos, slots, [first]]


@pytest.mark.parametrize("what", ["pages", "columns", "tokens", "negative"])
def test_page_tables_report_what_does_not_fit(what):
    page, cols, T, n_free = 16, 4, 100, 12
    old, new = [16, 10, 0], [20, 30, 17]   # 2 + 2 + 2 new pages from entry 3 on
    if what == "pages":
        n_free = 6
    if what == "columns":
        cols = 2
    if what == "tokens":
        T = 40
    if what == "negative":
        old[1], new[2] = -5, -9
    table = torch.full((3, 8), -1, dtype=torch.int32, device=DEV)  # columns from `cols` on are not the call's
    table[0, 0], table[1, 0] = 101, 102
    pos, slots = torch.full((T + 8,), -3, dtype=torch.int32, device=DEV), torch.full((T + 8,), -3, dtype=torch.int64, device=DEV)
    out = (i32([-3] * 4), i32([-3] * 3), pos[:T], slots[:T], i32([-3]))
    P.pifa_page_tables(i32(old), i32(new), page, i32(list(range(50, 50 + n_free))), i32([3]), table[:, :cols], T, out=out)
    assert P.pifa_device_status() == (P.PIFA_ERR_DEVICE_INDEX if what == "negative" else P.PIFA_ERR_CAPACITY)
    assert (table[:, cols:] == -1).all() and (pos[T:] == -3).all() and (slots[T:] == -3).all()
    got = slots[:T].tolist()
    if what == "pages":   # three of six pages: 53 for request 0, ...
        assert int(out[4]) == n_free and got[:20] == [53 * 16 + i for i in range(16)] + [54 * 16 + i for i in range(4)]
        assert got[20:26] == [102 * 16 + 10 + i for i in range(6)] and got[26:42] == [55 * 16 + i for i in range(16)]
        assert set(got[42:]) == {-1}
    if what == "columns":
        assert got[:16] == [53 * 16 + i for i in range(16)] and set(got[16:20]) == {-1}
    if what == "negative":
        assert out[0].tolist() == [0, 20, 50, 50] and out[1].tolist() == [36, 30, 0]


# ---- rotary positions ------------------------------------------------------------------------------------
def plain_rope(x, positions, freq, layout, scale=1.0, inverse=False):
    """float64; the phase from exact integers."""
    turns = torch.tensor([[(int(p) * int(f)) % 2 ** 64 / 2.0 ** 64 for f in freq.tolist()] for p in positions.tolist()],
                         dtype=torch.float64, device=DEV).view(len(positions), 1, -1)
    a = 2.0 * math.pi * turns * (-1.0 if inverse else 1.0)
    c, s, n = a.cos() * scale, a.sin() * scale, freq.numel()
    one, two = (slice(0, n), slice(n, 2 * n)) if layout == P.PIFA_ROPE_HALF else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    x = x.double()
    y, size = x.clone(), torch.zeros_like(x)
    y[..., one], y[..., two] = x[..., one] * c - x[..., two] * s, x[..., two] * c + x[..., one] * s
    size[..., one] = size[..., two] = (x[..., one].abs() + x[..., two].abs()) * abs(scale)
    return y, size


def check_rope(got, want, size, dtype):
    assert bool(((got.double() - want).abs() <= U[dtype] * want.abs() + 1e-6 * size + 2.0 ** -25).all())


LAYOUTS = [P.PIFA_ROPE_HALF, P.PIFA_ROPE_INTERLEAVED]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,h,d,rot", [(1, 1, 16, 16), (3, 5, 64, 64), (7, 32, 128, 128), (33, 3, 96, 32), (200, 9, 128, 48),
                                       (1, 64, 512, 512), (5000, 2, 64, 16)])
def test_rope_and_its_gradient(T, h, d, rot, dtype, layout):
    g = gen(T + d)
    X, dY = (torch.randn((T, h, d), device=DEV, generator=g).to(dtype) for _ in range(2))
    pos = torch.randint(0, 50000, (T,), device=DEV, generator=g).to(torch.int32)
    freq = P.pifa_rope_frequencies(rot, device=DEV)
    Y, dX = P.pifa_rope(X, pos, freq, layout), P.pifa_rope(dY, pos, freq, layout, inverse=True)
    for got, x, inv in ((Y, X, False), (dX, dY, True)):
        check_rope(got, *plain_rope(x, pos, freq, layout, inverse=inv), dtype)
    assert torch.equal(Y[..., rot:], X[..., rot:]) and torch.equal(dX[..., rot:], dY[..., rot:])
    # differences: the map is linear, so <dY, Y(X + E) - Y(X)> = <dX, E> but for the outputs' and X + E's roundings
    E = torch.randn((T, h, d), device=DEV, generator=g).to(dtype)
    XE = (X.double() + E.double()).to(dtype)
    YE = P.pifa_rope(XE, pos, freq, layout)
    lhs, rhs = (dY.double() * (YE.double() - Y.double())).sum(), (dX.double() * (XE.double() - X.double())).sum()
    slack = U[dtype] * ((dY.double() * YE.double()).abs().sum() + (dY.double() * Y.double()).abs().sum()
                        + (dX.double() * (XE.double() - X.double())).abs().sum())
    assert abs(float(lhs - rhs)) <= float(slack) * 1.01


@pytest.mark.parametrize("layout", LAYOUTS)
def test_rope_far_positions_strides_scale_and_place(layout):
    T, h, d = 9, 4, 128
    g = gen(3)
    whole = torch.randn((T, 3 * h, d), device=DEV, generator=g).to(torch.bfloat16)
    before = whole.clone()
    X = whole[:, h:2 * h]                                   # columns of a wider projection
    pos = i32([0, 1, 65535, 131071, 1000003, 2 ** 24 + 1, 2 ** 30 + 7, 2 ** 31 - 1, 17])
    freq = P.pifa_rope_frequencies(d, base=5e5, scaling=P.PIFA_ROPE_SCALE_BANDS, factor=8.0, original=8192.0, device=DEV)
    want, size = plain_rope(X, pos, freq, layout, scale=1.25)
    room = torch.full((T + 2, h * d + 24), 9.0, dtype=torch.bfloat16, device=DEV)
    Y = room[1:-1, 8:8 + h * d].unflatten(1, (h, d))
    P.pifa_rope(X, pos, freq, layout, scale=1.25, Y=Y)
    check_rope(Y, want, size, torch.bfloat16)
    assert (room[0] == 9).all() and (room[-1] == 9).all() and (room[:, :8] == 9).all() and (room[:, 8 + h * d:] == 9).all()
    assert P.pifa_rope(X, pos, freq, layout, scale=1.25, Y=X) is X and torch.equal(X, Y)   # in place
    assert torch.equal(whole[:, :h], before[:, :h]) and torch.equal(whole[:, 2 * h:], before[:, 2 * h:])


@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,hq,hk,d,rot,page", [(1, 1, 1, 64, 64, 16), (8, 32, 32, 128, 128, 16), (77, 14, 2, 64, 32, 13),
                                                (1300, 8, 8, 128, 128, 64), (6000, 3, 1, 96, 96, 128)])
def test_rope_cache(T, hq, hk, d, rot, page, dtype, heads_first):
    g = gen(T + hq)
    layout = LAYOUTS[T % 2]
    pages = T // page + 4
    qkv = torch.randn((T, hq + 2 * hk, d), device=DEV, generator=g).to(dtype)
    Q, K, V = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    pos = torch.randint(0, 9000, (T,), device=DEV, generator=g).to(torch.int32)
    freq = P.pifa_rope_frequencies(rot, device=DEV)
    slots = torch.randperm(pages * page, device=DEV, generator=g)[:T].contiguous()
    if T > 3:
        slots[2] = -1
    both = torch.full((pages, 2, hk, page, d) if heads_first else (pages, 2, page, hk, d), 7.0, dtype=dtype, device=DEV)
    kc, vc = both[:, 0], both[:, 1]                          # pages of keys and values in turn
    if heads_first:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    Qr = P.pifa_rope_cache(Q, K, V, pos, slots, freq, kc, vc, layout)
    check_rope(Qr, *plain_rope(Q, pos, freq, layout), dtype)
    kept = slots >= 0
    at = (slots[kept] // page, slots[kept] % page)
    want, size = plain_rope(K, pos, freq, layout)
    check_rope(kc[at], want[kept], size[kept], dtype)
    assert torch.equal(vc[at], V[kept])
    for c in (kc, vc):
        c[at] = 7.0
        assert (c == 7.0).all()
    kc2, vc2 = (torch.full((pages, page, hk, d), 7.0, dtype=dtype, device=DEV) for _ in range(2))
    assert P.pifa_rope_cache(Q, K, V, pos, slots, freq, kc2, vc2, layout, Qr=Q) is Q and torch.equal(Q, Qr)


def test_rope_cache_slots_outside_the_cache():
    T, h, d, page, pages = 5, 2, 64, 16, 3
    Q, K, V = (torch.ones((T, h, d), dtype=torch.bfloat16, device=DEV) for _ in range(3))
    room = torch.zeros((2, pages + 2, page, h, d), dtype=torch.bfloat16, device=DEV)
    slots = torch.tensor([0, pages * page, -2, 2 ** 40, pages * page - 1], device=DEV)
    P.pifa_rope_cache(Q, K, V, i32([0] * T), slots, P.pifa_rope_frequencies(d, device=DEV), room[0, 1:-1], room[1, 1:-1])
    assert P.pifa_device_status() == P.PIFA_ERR_DEVICE_INDEX
    assert int(room.sum()) == 2 * 2 * h * d and (room[:, 1, 0] == 1).all() and (room[:, -2, -1] == 1).all()


# ---- attention -------------------------------------------------------------------------------------------
def make_attention(seed, lens, news, hq, hk, d, page, dtype, heads_first=False, spare=0, dead=math.nan):
    """Requests over shuffled pages of a cache that holds `dead` wherever no request owns a token."""
    g = gen(seed)
    want = [-(-n // page) for n in lens]
    pages = sum(want) + 2 + spare
    shape = (pages, hk, page, d) if heads_first else (pages, page, hk, d)
    kc, vc = (torch.full(shape, dead, dtype=dtype, device=DEV) for _ in range(2))
    if heads_first:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    order = torch.randperm(pages, device=DEV, generator=g).tolist()
    cols = max(want + [1]) + 1
    table, at = torch.full((len(lens), cols), -1, dtype=torch.int32), 0
    for b, n in enumerate(lens):
        mine = order[at:at + want[b]]
        at += want[b]
        table[b, :want[b]] = torch.tensor(mine, dtype=torch.int32)
        for i, p in enumerate(mine):
            k = min(page, n - i * page)
            kc[p, :k] = torch.randn((k, hk, d), device=DEV, generator=g).to(dtype) * 1.5
            vc[p, :k] = torch.randn((k, hk, d), device=DEV, generator=g).to(dtype)
    start = [0]
    for n in news:
        start.append(start[-1] + n)
    Q = (torch.randn((start[-1], hq, d), device=DEV, generator=g) * 1.5).to(dtype)
    return dict(Q=Q, k_cache=kc, v_cache=vc, table=table.to(DEV), q_start=i32(start), kv_len=i32(lens))


def plain_attention(a, scale):
    """float64, request by request; also sum_j p_j |v_j| and the number of keys of each row."""
    Q, table = a["Q"].double(), a["table"]
    page, hk, d = a["k_cache"].shape[1:]
    G = Q.shape[1] // hk
    out, size, keys = torch.zeros_like(Q), torch.zeros_like(Q), torch.zeros(Q.shape[0], 1, 1, dtype=torch.float64, device=DEV)
    start, lens = a["q_start"].tolist(), a["kv_len"].tolist()
    for b, L in enumerate(lens):
        lo, hi = start[b], start[b + 1]
        if hi == lo or L == 0:
            continue
        rows = table[b, :-(-L // page)].long()
        k, v = (c[rows].flatten(0, 1)[:L].double().repeat_interleave(G, 1) for c in (a["k_cache"], a["v_cache"]))
        s = torch.einsum("qhd,khd->hqk", Q[lo:hi], k) * scale
        sees = torch.ones((hi - lo, L), dtype=torch.bool, device=DEV).tril(L - (hi - lo))
        p = torch.softmax(s.masked_fill(~sees, -math.inf), -1).nan_to_num(0.0)
        out[lo:hi], size[lo:hi] = torch.einsum("hqk,khd->qhd", p, v), torch.einsum("hqk,khd->qhd", p, v.abs())
        keys[lo:hi, 0, 0] = sees.sum(-1).double()
    return out, size, keys


def check_attention(a, O, scale):
    dtype = O.dtype
    want, size, keys = plain_attention(a, scale)
    tol = U[dtype] * (want.abs() + 1.1 * size) + 2e-4 * size
    if dtype is torch.float16:
        tol += 2.0 ** -24 * (1.0 + keys) * float(a["v_cache"].double().nan_to_num().abs().max())
    err = (O.double() - want).abs()
    assert bool((err <= tol).all()), (float((err - tol).max()), int((err > tol).sum()), (err > tol).nonzero()[:4].tolist())


def attend(a, max_q=None, scale=None, **kw):
    if max_q is None:
        max_q = max([1] + (a["q_start"][1:] - a["q_start"][:-1]).tolist())
    return P.pifa_paged_attention(a["Q"], a["k_cache"], a["v_cache"], a["table"], a["q_start"], a["kv_len"], max_q,
                                  scale=scale, **kw)


# (kv lengths, new tokens, query heads, kv heads, head_dim, page)
SHAPES = {
    "one_key": ([1], [1], 1, 1, 64, 16),
    "one_token": ([37], [1], 32, 32, 128, 16),
    "tokens_at_page_ends": ([15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 256, 257], [1] * 12, 4, 2, 128, 16),
    "decode_ragged_gqa": ([3000, 1, 700, 64, 2047], [1] * 5, 64, 8, 128, 64),
    "decode_group_7": ([500, 65], [1, 1], 14, 2, 64, 32),
    "decode_group_64": ([300, 90], [1, 1], 64, 1, 128, 128),
    "decode_long": ([40000], [1], 2, 1, 128, 256),
    "few_tokens": ([900, 17, 5, 333], [4, 2, 5, 3], 8, 8, 128, 16),
    "few_tokens_gqa": ([900, 4100, 5], [4, 2, 5], 16, 4, 64, 16),
    "prompt_odd": ([201], [201], 4, 4, 128, 16),
    "prompt_256": ([256], [256], 2, 1, 64, 64),
    "prompt_1000_gqa": ([1000], [1000], 6, 2, 128, 32),
    "chunk_in_context": ([2500], [300], 8, 2, 128, 64),
    "chunk_group_3": ([777, 130], [100, 130], 3, 1, 64, 16),
    "chunk_group_64": ([600], [65], 64, 1, 128, 16),
    "mixed": ([800, 45, 129, 2000, 300], [1, 45, 1, 257, 18], 8, 4, 128, 16),
    "rows_without_keys": ([5, 0, 64, 3], [9, 4, 64, 40], 4, 2, 128, 16),
    "no_new_tokens": ([70, 0, 40], [0, 0, 3], 4, 4, 64, 16),
    "many_requests": (list(range(1, 301)), [1 + b % 2 for b in range(300)], 2, 2, 64, 16),
}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", list(SHAPES))
def test_attention(name, dtype):
    lens, news, hq, hk, d, page = SHAPES[name]
    a = make_attention(len(name), lens, news, hq, hk, d, page, dtype)
    O = torch.full_like(a["Q"], math.nan)
    attend(a, O=O)
    check_attention(a, O, d ** -0.5)
    again = attend(a)
    assert torch.equal(again, O)     # and whatever order blocks run in


@pytest.mark.parametrize("name", ["tokens_at_page_ends", "few_tokens_gqa", "mixed", "prompt_1000_gqa"])
def test_attention_bound_on_new_tokens_may_be_loose(name):
    """A larger max_q may take another kernel: the same answer within the same bounds."""
    lens, news, hq, hk, d, page = SHAPES[name]
    a = make_attention(5, lens, news, hq, hk, d, page, torch.bfloat16)
    for loose in (16, 100, 5000):
        if loose >= max(news):
            check_attention(a, attend(a, max_q=loose), d ** -0.5)


@pytest.mark.parametrize("name", ["one_token", "few_tokens", "chunk_in_context", "mixed"])
def test_attention_strides_and_guards(name):
    """Heads before tokens in a page, queries as columns of a projection, padded outputs; rows of no request stay."""
    lens, news, hq, hk, d, page = SHAPES[name]
    a = make_attention(9, lens, news, hq, hk, d, page, torch.bfloat16, heads_first=True)
    T = a["Q"].shape[0]
    wide = torch.full((T + 3, hq + 5, d), 3.0, dtype=torch.bfloat16, device=DEV)
    wide[:T, 2:2 + hq] = a["Q"]
    a["Q"] = wide[:, 2:2 + hq]
    room = torch.full((T + 5, hq * d + 40), 9.0, dtype=torch.bfloat16, device=DEV)
    O = room[1:-1, 16:16 + hq * d].unflatten(1, (hq, d))
    attend(a, O=O)
    a["Q"] = a["Q"][:T]
    check_attention(a, O[:T], d ** -0.5)
    assert (room[0] == 9).all() and (room[T + 1:] == 9).all() and (room[:, :16] == 9).all() and (room[:, 16 + hq * d:] == 9).all()


@pytest.mark.parametrize("dead", [math.inf, -math.inf, math.nan, 6e4])
@pytest.mark.parametrize("name", ["tokens_at_page_ends", "few_tokens", "mixed"])
def test_attention_ignores_what_no_request_owns(name, dead):
    lens, news, hq, hk, d, page = SHAPES[name]
    for dtype in DTYPES:
        a = make_attention(2, lens, news, hq, hk, d, page, dtype, dead=dead)
        check_attention(a, attend(a), d ** -0.5) if dead != 6e4 else None
        b = make_attention(2, lens, news, hq, hk, d, page, dtype, dead=0.0)
        assert torch.equal(attend(a), attend(b))


@pytest.mark.parametrize("scale,size", [(1.0, 30.0), (-0.3, 2.0), (0.0, 1.0), (1e-3, 300.0)])
@pytest.mark.parametrize("name", ["decode_ragged_gqa", "prompt_1000_gqa"])
def test_attention_scores_of_any_size(name, scale, size):
    """Scores in the hundreds (one key takes all), negative scales, equal scores. Scores of size S carry fp32
    errors of 2^-23 S sqrt(d) or so, within 1e-3 of a weight here."""
    lens, news, hq, hk, d, page = SHAPES[name]
    a = make_attention(3, lens, news, hq, hk, d, page, torch.bfloat16)
    a["Q"] = (a["Q"].float() * size / 1.5).to(torch.bfloat16)
    O = attend(a, scale=scale)
    want, s, _ = plain_attention(a, scale)
    assert bool(((O.double() - want).abs() <= U[torch.bfloat16] * (want.abs() + 1.1 * s) + 2e-3 * s + 1e-6).all())


@pytest.mark.parametrize("new", [1, 3, 200])
def test_attention_offsets_past_32_bits(new):
    """A cache of 5 Gi elements, its requests' pages at both ends."""
    hq, hk, d, page, L = 4, 2, 128, 64, 700
    a = make_attention(1, [L, 300], [new, 1], hq, hk, d, page, torch.bfloat16)
    pages = 5 * 2 ** 30 // (page * hk * d)
    used = a["k_cache"].shape[0]
    for name in ("k_cache", "v_cache"):
        big = torch.empty((pages, page, hk, d), dtype=torch.bfloat16, device=DEV)
        big[pages - used:] = a[name]
        a[name] = big
    a["table"] = torch.where(a["table"] >= 0, a["table"] + (pages - used), -1)
    lo = int(a["table"][0, 1])                       # one page at the other end
    for name in ("k_cache", "v_cache"):
        a[name][0] = a[name][lo]
    a["table"][0, 1] = 0
    O = attend(a)
    rows = a["table"].clamp(min=0).long()
    small = dict(a, k_cache=a["k_cache"][rows].flatten(0, 1), v_cache=a["v_cache"][rows].flatten(0, 1),
                 table=torch.arange(rows.numel(), device=DEV, dtype=torch.int32).view(rows.shape))
    check_attention(small, O, d ** -0.5)


def test_attention_reports_bad_tables_and_bounds():
    for new in (1, 40):
        a = make_attention(7, [200, 90], [new, 1], 4, 2, 128, 16, torch.bfloat16)
        good = attend(a)
        for bad in (-1, 10 ** 6, 2 ** 31 - 1):
            b = dict(a, table=a["table"].clone())
            b["table"][0, 3] = bad
            O = attend(b)
            assert P.pifa_device_status() == P.PIFA_ERR_DEVICE_INDEX
            assert torch.equal(O[new:], good[new:])            # the other request's
            z = dict(a, k_cache=a["k_cache"].clone(), v_cache=a["v_cache"].clone())
            z["k_cache"][int(a["table"][0, 3])] = 0.0
            z["v_cache"][int(a["table"][0, 3])] = 0.0
            check_attention(z, O, 128 ** -0.5)
        b = dict(a, kv_len=i32([10 ** 6, 90]))
        O = attend(b)
        assert P.pifa_device_status() in (P.PIFA_ERR_CAPACITY, P.PIFA_ERR_DEVICE_INDEX)
        check_attention(a, torch.cat([good[:new], O[new:]]), 128 ** -0.5)   # other lengths, other cuts of the work
    O = torch.full_like(a["Q"], 5.0)
    attend(a, max_q=3, O=O)
    assert P.pifa_device_status() == P.PIFA_ERR_CAPACITY
    assert (O[3:40] == 5.0).all()
    check_attention(dict(a, Q=a["Q"]), torch.cat([O[:3], good[3:40], O[40:]]), 128 ** -0.5)


def test_attention_in_a_graph_and_on_a_stream():
    """Captured once with room for any lengths, replayed after the lengths, tables and cache changed."""
    hq, hk, d, page = 8, 2, 128, 16
    a = make_attention(11, [500, 33, 64], [1, 1, 1], hq, hk, d, page, torch.bfloat16)
    b = make_attention(12, [40, 480, 77], [1, 1, 1], hq, hk, d, page, torch.bfloat16)
    for x in (a, b):  # one size of cache and table
        x["table"] = torch.nn.functional.pad(x["table"], (0, 64 - x["table"].shape[1]), value=-1).contiguous()
        for name in ("k_cache", "v_cache"):
            x[name] = torch.cat([x[name], x[name].new_full((90 - x[name].shape[0], page, hk, d), math.nan)])
    O, ws = torch.empty_like(a["Q"]), torch.empty(P.pifa_paged_attention_workspace_size(3, hq, hk, d, 3, 1) + 256,
                                                  dtype=torch.uint8, device=DEV)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    attend(a, max_q=1, O=O, workspace_tensor=ws, stream=stream)
    stream.synchronize()
    check_attention(a, O, d ** -0.5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        attend(a, max_q=1, O=O, workspace_tensor=ws, stream=stream)
    for name in a:
        a[name].copy_(b[name])
    O.fill_(math.nan)
    graph.replay()
    torch.cuda.synchronize()
    check_attention(b, O, d ** -0.5)
    with torch.cuda.stream(stream):
        O2 = attend(b)
    stream.synchronize()
    assert torch.equal(O, O2)


@pytest.mark.parametrize("width,heads", [(512, 4), (1024, 16)])
def test_the_example_serves_prompts_and_decode_steps(width, heads):
    """PIFA projections, page tables, rotation with the cache write and attention together, the decode step as a replayed
    graph. The bf16 values between the calls (x, q, k, v, o) carry relative errors of 2^-9 rms each: within 4%
    of the outputs' rms at the largest of some thousands of elements (4.5 sigma of about 2^-7)."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_block.py")
    spec = importlib.util.spec_from_file_location("attention_block", path)
    block = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(block)
    error, _, _ = block.serve(width=width, heads=heads, requests=5, prompt=83, steps=20)
    assert error < 0.04


def test_attention_on_two_streams_at_once():
    """Calls on two streams overlap, each with its own scratch: the same bits as one after the other."""
    hq, hk, d, page = 16, 4, 128, 32
    sets = [make_attention(21, [3000, 40, 700], [300, 1, 77], hq, hk, d, page, torch.bfloat16),
            make_attention(22, [9000, 5000], [1, 1], hq, hk, d, page, torch.bfloat16),
            make_attention(23, [6000], [70], hq, hk, d, page, torch.bfloat16),
            make_attention(24, [200] * 40, [3] * 40, hq, hk, d, page, torch.bfloat16)]
    bounds = [300, 1, 70, 3]
    serial = [attend(a, max_q=n) for a, n in zip(sets, bounds)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for k in range(24):
        for s in (0, 1):
            with torch.cuda.stream(streams[s]):
                i = (k + 2 * s) % 4
                got[s].append((i, attend(sets[i], max_q=bounds[i])))
    torch.cuda.synchronize()
    for s in (0, 1):
        for i, O in got[s]:
            assert torch.equal(O, serial[i])
