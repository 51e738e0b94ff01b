"""Attention over a cache in 8 bits, path by path: long requests whose every piece is visible in the output, heads that are cut and
not cut, waits that run out, graphs captured with the default scratch."""
import math

import pytest
import torch

from paper_2501_19090_gb300 import pifa as P
from test_attention_pieces import SHAPES, U, check_counts, counts, hot
from test_attention_timeout_gpu import SHAPES as CHUNKS
from test_cache_q8_gpu import E4M3, E8M0, U8, attend, check_attention, empty_cache, make_q8, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = [torch.bfloat16, torch.float16]


def quantised(a, K, V):
    """The cache of dense keys and values (tokens of all requests in a row), NaN where no request owns a token."""
    pages, page, hk, d = a["pages"], a["page"], a["hk"], K.shape[2]
    cache = empty_cache(pages, page, hk, d)
    for i, x in enumerate((K, V)):
        full = torch.zeros((pages * page, hk, d), dtype=torch.float64, device=DEV)
        full[a["slots"]] = x.double()
        blocks = full.view(pages, page // 16, 16, hk, d)
        e = torch.ceil(torch.log2(blocks.abs().amax((2, 4)).clamp(min=2.0 ** -100) / 448.0) - 1e-9)
        q = (blocks * torch.exp2(-e)[:, :, None, :, None]).float().clamp(-448, 448).to(E4M3).view(U8).view(pages * page, hk, d)
        at = a["slots"]
        cache[i].view(U8)[at // page, at % page] = q[at]
        cache[2 + i].view(U8)[at // page, at % page // 16] = (e + 127).to(U8)[at // page, at % page // 16]
    return cache


def run(a, cache, room):
    O = torch.full_like(a["Q"], math.nan)
    x = dict(Q=a["Q"], k8=cache[0], v8=cache[1], ks=cache[2], vs=cache[3], table=a["table"], q_start=a["q_start"], kv_len=a["kv_len"])
    attend(x, max_q=max(a["news"]), O=O, room=room)
    assert P.pifa_device_status() == P.PIFA_OK
    return O


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", list(SHAPES))
def test_every_piece_is_counted_once(name, dtype, room):
    """Values of one are held exactly, so the bounds are those of a cache in 16 bits."""
    a, K, V, want = counts(name, dtype, DEV)
    assert check_counts(run(a, quantised(a, K, V), room), want, dtype)


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", list(SHAPES))
def test_every_piece_can_hold_the_largest_score(name, dtype, room):
    """The key of the largest score keeps it, but for e4m3's rounding (56 at least), and the others keep scores of zero."""
    for seed in range(6):
        a, K, V, keys, _ = hot(name, dtype, DEV, seed)
        cache = quantised(a, K, V)
        v = values(cache[1], cache[3])
        want = torch.empty(a["Q"].shape, dtype=torch.float64, device=DEV)
        G, row, first = a["Q"].shape[1] // a["hk"], 0, 0
        for b, (L, n) in enumerate(zip(a["lens"], a["news"])):
            for h in range(a["hk"]):
                slot = int(a["slots"][first + keys[b][h]])
                want[row:row + n, h * G:(h + 1) * G] = v[slot // a["page"], slot % a["page"], h]
            row, first = row + n, first + L
        got = run(a, cache, room)
        tol = 2.02 * U[dtype] * want.abs() + 2e-10 + 2.0 ** -24 * float(v[a["slots"] // a["page"], a["slots"] % a["page"]].abs().max())
        assert bool(((got.double() - want).abs() <= tol).all()), seed


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq,hk,d", [(32, 32, 128), (16, 2, 64), (8, 1, 128)])
@pytest.mark.parametrize("lens", [[1], [16, 17, 0, 5], [500, 3, 64, 511, 129], list(range(1, 160))])
def test_heads_that_are_not_cut(lens, hq, hk, d, dtype):
    """A table with room for few keys leaves heads whole; one with more columns cuts them: the same rows within the same bounds."""
    news = [1 if n else 0 for n in lens]
    a = make_q8(31, lens, news, hq, hk, d, 16, dtype)
    for cols in (a["table"].shape[1], 40, 500):
        b = dict(a, table=torch.nn.functional.pad(a["table"], (0, cols - a["table"].shape[1]), value=-1).contiguous()
                 if cols > a["table"].shape[1] else a["table"])
        O = torch.full_like(a["Q"], math.nan)
        attend(b, max_q=1, O=O)
        check_attention(b, O, d ** -0.5)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hk,new", [(1, 1, 1), (7, 1, 1), (16, 2, 1), (18, 2, 1), (4, 2, 3), (5, 1, 3), (2, 1, 8), (16, 1, 1), (1, 1, 16)])
def test_heads_that_are_cut(hq, hk, new, d):
    """One to sixteen rows a key / value head, heads in two pieces and in many, beside short ones and one without keys."""
    lens = [9000, 17, 0, 300, 2500, 16, 40000]
    news = [min(new, n) for n in lens]
    for pick in (slice(0, 7), slice(6, 7), slice(1, 5)):
        a = make_q8(32, lens[pick], news[pick], hq, hk, d, 64, torch.bfloat16)
        O = torch.full_like(a["Q"], math.nan)
        attend(a, max_q=new, O=O)
        check_attention(a, O, d ** -0.5)
        again = attend(a, max_q=new, O=torch.full_like(O, math.nan))
        assert torch.equal(O, again)


@pytest.mark.parametrize("B", [511, 513, 4096])
@pytest.mark.parametrize("cols", [None, 700])
def test_many_requests(B, cols):
    """More requests than there are CTAs, threads of one, and lengths that it keeps at hand; the long ones last."""
    lens = [(7 * b * b + 3 * b) % 90 for b in range(B - 3)] + [2000, 1, 3000]
    a = make_q8(33, lens, [min(n, 1) for n in lens], 4, 2, 128, 16, torch.float16)
    if cols:
        a = dict(a, table=torch.nn.functional.pad(a["table"], (0, cols - a["table"].shape[1]), value=-1).contiguous())
    O = torch.full_like(a["Q"], math.nan)
    attend(a, max_q=1, O=O)
    check_attention(a, O, 128 ** -0.5)


@pytest.fixture
def _bound():
    yield
    P.pifa_set_wait_timeout(0)
    P.pifa_device_status()


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("name", list(CHUNKS))
def test_waits_that_run_out(name, room, _bound):
    lens, news, hq, hk, d, page = CHUNKS[name]
    a = make_q8(6, lens, news, hq, hk, d, page, torch.bfloat16)
    T = a["Q"].shape[0]
    frame = torch.full((T + 2, hq, d), 9.0, dtype=torch.bfloat16, device=DEV)
    want = attend(a, O=torch.empty_like(a["Q"]), room=room)
    assert P.pifa_device_status() == P.PIFA_OK
    check_attention(a, want, d ** -0.5)
    for ns in (1, 1, 500, 2000, 5000, 10000, 20000):
        P.pifa_set_wait_timeout(ns)
        attend(a, O=frame[1:-1], room=room)
        status = P.pifa_device_status()
        assert status == P.PIFA_ERR_TIMEOUT or (ns > 1 and status == P.PIFA_OK)
        assert bool((frame[0] == 9.0).all() and (frame[-1] == 9.0).all())
        P.pifa_set_wait_timeout(0)
        O = attend(a, O=torch.full_like(want, math.nan), room=room)
        assert P.pifa_device_status() == P.PIFA_OK and torch.equal(O, want)


@pytest.mark.parametrize("news,lens", [([1, 1, 1], [2000, 33, 64]), ([40, 1], [900, 300]), ([500, 2], [900, 300])])
def test_graph_with_default_scratch(news, lens):
    """Captured twice in a row on a stream, then larger eager calls on it: replays neither change what lies over the scratch that
    those gave back nor are changed, also beside an eager call."""
    hq, hk, d, page = 8, 2, 128, 16
    a = make_q8(31, lens, news, hq, hk, d, page, torch.bfloat16)
    big = make_q8(32, [1500, 700], [900, 700], hq, hk, d, page, torch.bfloat16)
    want, big_want = attend(a), attend(big)
    O, big_O = torch.empty_like(a["Q"]), torch.empty_like(big["Q"])
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            attend(a, max_q=max(news), O=O)
            attend(a, max_q=max(news), O=O)
        attend(big, max_q=900, O=big_O)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        fill = [torch.full((n,), 77, dtype=U8, device=DEV) for n in (2 ** 20, 2 ** 22, 2 ** 24, 2 ** 26) * 4]
    O.fill_(math.nan)
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(O, want) and all(bool((x == 77).all()) for x in fill)
    for _ in range(20):
        with torch.cuda.stream(other):
            graph.replay()
        with torch.cuda.stream(stream):
            attend(big, max_q=900, O=big_O)
    torch.cuda.synchronize()
    assert torch.equal(O, want) and torch.equal(big_O, big_want)


def test_room_is_guarded():
    """Scratch of exactly the bytes asked for, between guard bytes, for each path; O inside the room for 16 bits is refused."""
    for lens, news, hq, hk, d in (([900, 20], [1, 1], 8, 2, 128), ([900, 20], [70, 1], 8, 2, 128), ([900, 20], [500, 1], 8, 2, 128)):
        a = make_q8(5, lens, news, hq, hk, d, 32, torch.bfloat16)
        B, cols = a["table"].shape
        need = P.pifa_paged_attention_q8_workspace_size(a["Q"].shape[0], hq, hk, d, B, max(news), cols, 32)
        ws = torch.full((need + 1024,), 0x5a, dtype=U8, device=DEV)
        lo = -ws.data_ptr() % 256 + 256
        O = P.pifa_paged_attention_q8(a["Q"], a["k8"], a["v8"], a["ks"], a["vs"], a["table"], a["q_start"], a["kv_len"], max(news),
                                      workspace_tensor=ws[lo:lo + need])
        assert torch.equal(O, attend(a)) and (ws[:lo] == 0x5a).all() and (ws[lo + need:] == 0x5a).all()
    inside = ws[lo + need - O.numel() * 2:lo + need]
    inside = inside[-inside.data_ptr() % 16:]
    with pytest.raises(P.PifaError, match="overlaps"):
        P.pifa_paged_attention_q8(a["Q"][:-60], a["k8"], a["v8"], a["ks"], a["vs"], a["table"], a["q_start"], a["kv_len"], max(news),
                                  O=inside[:a["Q"][:-60].numel() * 2].view(torch.bfloat16).view(a["Q"][:-60].shape), workspace_tensor=ws[lo:lo + need])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 96, 128, 256, 512])
def test_write_of_many_tokens_equals_that_of_few(d, dtype):
    """A prompt in one call (its own form of the kernel) and in calls of some hundred tokens: the same bytes, but for what is rounded
    twice in the subnormal range."""
    T, hk, page = 2500, 2, 64
    g = torch.Generator(device=DEV).manual_seed(d)
    x = torch.randn((T, 3 * hk, d), device=DEV, generator=g)
    x[:, hk:] *= torch.exp2(torch.randint(-3, 4, (T, 2 * hk, 1), device=DEV, generator=g).float())
    Q, K, V = x.to(dtype).split(hk, 1)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    order = torch.randperm(45, device=DEV, generator=g)
    slots = order[(pos.long() + 5) // page] * page + (pos.long() + 5) % page
    freq = P.pifa_rope_frequencies(d, device=DEV)
    one, many = empty_cache(45, page, hk, d), empty_cache(45, page, hk, d)
    for c in (one, many):                              # the first block holds five tokens already
        P.pifa_rope_cache_q8(Q[:5], K[:5], V[:5], pos[:5], order[0] * page + torch.arange(5, device=DEV), freq, *c)
    Qr = P.pifa_rope_cache_q8(Q, K, V, pos, slots, freq, *one)
    parts = [P.pifa_rope_cache_q8(Q[i:i + 700], K[i:i + 700], V[i:i + 700], pos[i:i + 700], slots[i:i + 700], freq, *many) for i in range(0, T, 700)]
    assert torch.equal(Qr, torch.cat(parts)) and torch.equal(Qr, P.pifa_rope(Q, pos, freq))
    for i in (0, 1):
        assert torch.equal(one[2 + i].view(U8), many[2 + i].view(U8))
        a, b = one[i].double().nan_to_num(0.0), many[i].double().nan_to_num(0.0)
        assert torch.equal(one[i].double().isnan(), many[i].double().isnan())
        assert bool(((a == b) | (((a - b).abs() <= 2.0 ** -9) & (b.abs() <= 2.0 ** -6))).all())


@pytest.mark.parametrize("hq,hk,d", [(64, 8, 128), (32, 32, 128), (40, 5, 64), (3, 1, 512)])
@pytest.mark.parametrize("T", [33, 64, 100, 181, 200, 303, 607])
def test_tokens_of_many_requests_equal_those_of_few(T, hq, hk, d):
    """However tokens, heads and queries are dealt to CTAs: the bytes of the cache, and the queries, are those of calls of eight tokens."""
    g = torch.Generator(DEV).manual_seed(T + hq)
    x = torch.randn((T, hq + 2 * hk, d), device=DEV, generator=g)
    x[:, hq:] *= torch.exp2(torch.randint(-6, 7, (T, 2 * hk, 1), device=DEV, generator=g).float())
    x = x.to(torch.bfloat16)
    Q, K, V = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    at = torch.randperm(T, device=DEV, generator=g) * 16 + torch.randint(0, 16, (T,), device=DEV, generator=g)  # a block each
    pos = torch.randint(0, 100000, (T,), device=DEV, generator=g).int()
    freq = P.pifa_rope_frequencies(d // 2, device=DEV)
    one = empty_cache((T + 3) // 4, 64, hk, d, byte=0x35)
    one[2].view(U8).random_(110, 140, generator=g)
    one[3].view(U8).random_(110, 140, generator=g)
    all_at_once = [c.clone() for c in one]
    want = torch.cat([P.pifa_rope_cache_q8(Q[i:i + 8], K[i:i + 8], V[i:i + 8], pos[i:i + 8], at[i:i + 8], freq, *one) for i in range(0, T, 8)])
    got = P.pifa_rope_cache_q8(Q, K, V, pos, at, freq, *all_at_once)
    assert P.pifa_device_status() == P.PIFA_OK
    assert torch.equal(got, want) and torch.equal(got, P.pifa_rope(Q, pos, freq))
    for a, b in zip(one, all_at_once):
        assert torch.equal(a.view(U8), b.view(U8))


def test_calls_of_nothing():
    cache = empty_cache(3, 16, 2, 64)
    e = torch.empty
    none = dict(dtype=torch.bfloat16, device=DEV)
    i32, i64 = torch.int32, torch.int64
    freq = P.pifa_rope_frequencies(64, device=DEV)
    Qr = P.pifa_rope_cache_q8(e((0, 4, 64), **none), e((0, 2, 64), **none), e((0, 2, 64), **none), e(0, dtype=i32, device=DEV),
                              e(0, dtype=i64, device=DEV), freq, *cache)
    K, V = P.pifa_cache_read_q8(*cache, e(0, dtype=i64, device=DEV))
    assert Qr.shape == (0, 4, 64) and K.shape == V.shape == (0, 2, 64)
    O = torch.full((3, 4, 64), 5.0, **none)
    P.pifa_paged_attention_q8(O.clone(), *cache, e((0, 4), dtype=i32, device=DEV), torch.zeros(1, dtype=i32, device=DEV), e(0, dtype=i32, device=DEV), 1, O=O)
    P.pifa_paged_attention_q8(O[:0], *cache, e((2, 4), dtype=i32, device=DEV), torch.zeros(3, dtype=i32, device=DEV), torch.zeros(2, dtype=i32, device=DEV), 1)
    assert (O == 5.0).all() and (cache[0].view(U8) == 0x7f).all()
    for new in (2, 40, 900):                           # a table without columns: no keys
        O = P.pifa_paged_attention_q8(torch.ones((new, 4, 64), **none), *cache, e((1, 0), dtype=i32, device=DEV),
                                      torch.tensor([0, new], dtype=i32, device=DEV), torch.zeros(1, dtype=i32, device=DEV), new)
        assert (O == 0).all()


@pytest.mark.parametrize("width,heads", [(512, 4), (1024, 16)])
def test_the_example_serves_from_a_cache_in_8_bits(width, heads):
    """It runs. An e4m3 number is off by 2^-4 at most, so values of up to 4.5 times the rms by 0.28 of it; the outputs, their sums with
    weights that add up to one, by less, and those of projections of some hundred such sums by about as much: under half."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_block.py")
    spec = importlib.util.spec_from_file_location("attention_block", path)
    block = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(block)
    error, _, _ = block.serve(width=width, heads=heads, requests=5, prompt=83, steps=20, cache_bits=8)
    assert error < 0.5
