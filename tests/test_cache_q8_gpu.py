"""GPU parity of the paged cache in 8 bits: written, read back and attended to, each against 64 bits.

Bounds:
  write       scales are whole exponents and have to be those of the exact values, or of values 1e-6 away. An element stands for a
              value within half an e4m3 step of the exact one, max(2^-4 |x|, 2^-10 s), and 1e-6 (|x| + |partner|) for the rotation
              in fp32. Elements that a call keeps are rounded anew to a scale 2^k higher: e4m3's rounding of q / 2^k, exactly.
  read        element times scale, rounded once: exact in bf16, u |x| + 2^-25 in fp16
  attention   of the values that the cache stands for. Weights are fp16 (of long chunks that are brought to 16 bits first, dtype: w) and
              the output is rounded once: u |o| + w sum p |v| (first order, 10% over for the rest), 2e-4 sum p |v| for fp32
              scores, exponentials and sums, and 2^-24 max |v| a
              key, for weights below fp16's normal range: a weight, times its value's scale, is held relative to the largest of them,
              which is at least 1 there, so its error of 2^-25 times an element of at most 448 is at most 2^-24 max |v| in the sum.
              Q in fp16 is exact but for elements less than 2^-28 of their row's largest.
"""
import math
import random

import pytest
import torch

from paper_2501_19090_gb300 import pifa as P
from test_attention_path_gpu import SHAPES, gen, i32, make_attention, plain_attention, plain_rope

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
DTYPES = [torch.bfloat16, torch.float16]
E4M3, E8M0, U8 = torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.uint8


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    P.load()
    yield


@pytest.fixture(autouse=True)
def _clean_status():
    yield
    assert P.pifa_device_status() == P.PIFA_OK  # a test that expects an error has read it


# ---- caches ----------------------------------------------------------------------------------------------
def empty_cache(pages, page, hk, d, heads_first=False, byte=0x7f):
    """Elements and scales that nobody has written: NaN (or any byte)."""
    shape = (pages, 2, hk, page, d) if heads_first else (pages, 2, page, hk, d)
    both = torch.full(shape, byte, dtype=U8, device=DEV)          # pages of keys and values in turn
    k, v = both[:, 0], both[:, 1]
    if heads_first:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
        s = torch.full((2, hk, pages, page // 16), 0xff, dtype=U8, device=DEV).permute(0, 2, 3, 1)
    else:
        s = torch.full((2, pages, page // 16, hk), 0xff, dtype=U8, device=DEV)
    return [k.view(E4M3), v.view(E4M3), s[0].view(E8M0), s[1].view(E8M0)]


def values(cache, scale):
    """What a cache stands for, float64, pages x page x heads x d."""
    return cache.double() * scale.double().repeat_interleave(16, 1)[..., None]


def exponent(a):
    """Of the smallest power of two with a <= 448 2^e, on the host, from -126 on."""
    if a == 0.0:
        return -126
    m, e = math.frexp(a)
    return max(e - 9 if m <= 0.875 else e - 8, -126)


def blocks_of(slots):
    """{block: [(offset, row)]} of a call's slots."""
    out = {}
    for t, s in enumerate(slots.tolist()):
        if s >= 0:
            out.setdefault(s // 16, []).append((s % 16, t))
    return out


def check_store(before, after, scales_before, scales_after, x, size, slots, page):
    """One of the two caches after a call that wrote x (float64, T x heads x d) at slots; all in bytes but x and size."""
    hk, d = x.shape[1:]
    flat = lambda c: c.contiguous().view(-1, 16, hk, d)
    b8, a8 = flat(before.view(U8)), flat(after.view(U8))
    sb, sa = (s.view(U8).contiguous().view(-1, hk).tolist() for s in (scales_before, scales_after))
    want8, seen = b8.clone(), torch.zeros(b8.shape[0], dtype=torch.bool)
    for blk, rows in blocks_of(slots).items():
        seen[blk] = True
        offs, ts = [o for o, _ in rows], [t for _, t in rows]
        mag = torch.where(x[ts].isfinite(), x[ts].abs(), 0.0).amax((0, 2)).tolist()
        slack = size[ts].amax((0, 2)).tolist()
        for h in range(hk):
            got, was = sa[blk][h], sb[blk][h]
            lo, hi = exponent(max(mag[h] - 1e-6 * slack[h], 0.0)) + 127, exponent(mag[h] + 1e-6 * slack[h]) + 127
            if min(offs) > 0:
                lo, hi = max(lo, was), max(hi, was)
            assert lo <= got <= hi, (blk, h, got, lo, hi, was)
            want8[blk, offs, h] = a8[blk, offs, h]               # checked as values below
            if min(offs) > 0 and got > was:
                f = 2.0 ** (was - got)
                rest = [o for o in range(16) if o not in offs]
                want8[blk, rest, h] = (b8[blk, rest, h].view(E4M3).double() * f).to(E4M3).view(U8)
    nan = lambda c: (c & 0x7f) == 0x7f
    assert bool(((a8 == want8) | (nan(a8) & nan(want8))).all())
    kept = [t for t, s in enumerate(slots.tolist()) if s >= 0]
    at = slots[kept]
    q, s = a8.view(-1, hk, d)[at].view(E4M3).double(), torch.tensor(sa, device=DEV).view(-1, hk)[at // 16].double()
    s = torch.exp2(s - 127)[..., None]
    w = x[kept]
    fine = w.isfinite()
    assert bool((q.isnan() == ~fine).all())
    err, tol = (q * s - w).abs(), torch.maximum(2.0 ** -4 * w.abs(), 2.0 ** -10 * s) * (1 + 1e-9) + 1e-6 * size[kept]
    assert bool((err <= tol)[fine].all()), float((err - tol)[fine].max())
    changed = (torch.tensor(sa) != torch.tensor(sb)).any(1)
    assert bool((~changed | seen).all())                          # scales of other blocks


def steps(rng, B, page, most_old, most_new):
    """Requests that hold `old` tokens and get `new` ones: (old, new, slots of all their tokens)."""
    old = [rng.choice([0, 16, rng.randint(0, most_old)]) for _ in range(B)]
    new = [rng.choice([1, 1, rng.randint(0, most_new)]) for _ in range(B)]
    pages = list(range(sum(-(-(o + n) // page) for o, n in zip(old, new)) + 3))
    rng.shuffle(pages)
    slots = []
    for o, n in zip(old, new):
        mine = [pages.pop() for _ in range(-(-(o + n) // page))]
        slots.append([mine[i // page] * page + i % page for i in range(o + n)])
    return old, new, slots


def write(x, pos, slots, freq, cache, layout=P.PIFA_ROPE_HALF, **kw):
    Q, K, V = x
    return P.pifa_rope_cache_q8(Q, K, V, pos, slots, freq, *cache, layout, **kw)


def inputs(g, T, hq, hk, d, dtype, sizes=(1.0, 1.0)):
    """Columns of one projection's output; keys and values whose size changes from token to token."""
    x = torch.randn((T, hq + 2 * hk, d), device=DEV, generator=g)
    x[:, hq:] *= torch.exp2(torch.randint(-4, 5, (T, 2 * hk, 1), device=DEV, generator=g).float())
    x[:, hq:hq + hk] *= sizes[0]
    x[:, hq + hk:] *= sizes[1]
    x = x.to(dtype)
    return x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]


# ---- writing -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,most_old,most_new,hq,hk,d,rot,page", [
    (1, 0, 1, 1, 1, 64, 64, 16), (8, 100, 1, 32, 32, 128, 128, 16), (40, 300, 20, 14, 2, 64, 32, 48), (3, 40, 700, 8, 8, 128, 128, 64),
    (5, 90, 60, 3, 1, 96, 96, 128), (4, 50, 33, 2, 3, 256, 64, 32), (3, 20, 40, 2, 2, 512, 512, 16), (2, 30, 18, 1, 1, 16, 16, 16),
    (2, 7, 1500, 4, 1, 144, 48, 256), (300, 50, 1, 8, 8, 128, 128, 64)])
def test_write(B, most_old, most_new, hq, hk, d, rot, page, dtype, heads_first):
    rng, g = random.Random(B * d + most_new), gen(B + d)
    layout = [P.PIFA_ROPE_HALF, P.PIFA_ROPE_INTERLEAVED][(B + d // 16) % 2]
    old, new, slots = steps(rng, B, page, most_old, most_new)
    pages = max([0] + [s // page for r in slots for s in r]) + 2
    cache, freq = empty_cache(pages, page, hk, d, heads_first), P.pifa_rope_frequencies(rot, device=DEV)
    for which in (0, 1):                       # the tokens that are held, then the new ones
        part = [r[:o] if which == 0 else r[o:] for r, o in zip(slots, old)]
        at = torch.tensor([s for r in part for s in r] + [-1, -1], dtype=torch.int64, device=DEV)  # rows behind the last token
        pos = i32([i + (0 if which == 0 else o) for r, o in zip(part, old) for i in range(len(r))] + [0, 0])
        Q, K, V = inputs(g, len(at), hq, hk, d, dtype, sizes=(3.0, 0.2) if which else (1.0, 1.0))
        before = [c.clone() for c in cache]
        Qr = write((Q, K, V), pos, at, freq, cache, layout, scale=1.0 if B != 5 else 1.25)
        turned, size = plain_rope(K, pos, freq, layout, scale=1.0 if B != 5 else 1.25)
        check_store(before[0], cache[0], before[2], cache[2], turned, size, at, page)
        check_store(before[1], cache[1], before[3], cache[3], V.double(), torch.zeros_like(size), at, page)
        same = P.pifa_rope(Q, pos, freq, layout, scale=1.0 if B != 5 else 1.25)
        assert torch.equal(Qr, same)           # the queries are pifa_rope's
    assert write((Q, K, V), pos, at, freq, cache, layout, scale=1.0 if B != 5 else 1.25, Qr=Q) is Q and torch.equal(Q, Qr)  # in place


@pytest.mark.parametrize("d", [64, 256])
def test_token_by_token_gives_the_scales_of_a_whole_prompt(d):
    T, hk, page = 100, 3, 32
    g, freq = gen(d), P.pifa_rope_frequencies(d, device=DEV)
    x = inputs(g, T, 2, hk, d, torch.bfloat16)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    slots = torch.tensor([5, 1, 7, 2], device=DEV)[pos.long() // page] * page + pos.long() % page
    whole, one, odd = (empty_cache(9, page, hk, d) for _ in range(3))
    write(x, pos, slots, freq, whole)
    for t in range(T):
        write([y[t:t + 1] for y in x], pos[t:t + 1], slots[t:t + 1], freq, one)
    cuts = [0, 3, 20, 21, 37, 64, 95, T]
    for a, b in zip(cuts, cuts[1:]):
        write([y[a:b] for y in x], pos[a:b], slots[a:b], freq, odd)
    at = (slots // page, slots % page)
    for c in (one, odd):
        for i in (0, 1):
            assert torch.equal(c[2 + i].view(U8)[slots // page, slots % page // 16], whole[2 + i].view(U8)[slots // page, slots % page // 16])
            # elements that were rounded more than once differ by a step of the subnormal range at most
            a, b = c[i][at].double(), whole[i][at].double()
            assert bool(((a == b) | (((a - b).abs() <= 2.0 ** -9) & (b.abs() <= 2.0 ** -6))).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinities_and_nan_leave_the_scale_to_the_others(dtype):
    T, hk, d, page = 40, 2, 128, 16
    g, freq = gen(1), P.pifa_rope_frequencies(d, device=DEV)
    Q, K, V = (y.clone() for y in inputs(g, T, 1, hk, d, dtype))
    for t, h, e, x in ((0, 0, 3, math.inf), (3, 1, 127, -math.inf), (17, 0, 64, math.nan), (39, 1, 0, math.nan)):
        V[t, h, e] = x
        K[t, h, e] = x
    V[20, 0] = math.nan                                        # a whole token
    K[20, 0] = math.inf
    slots, pos = torch.arange(T, device=DEV) + 16, i32([0] * T)  # position 0: nothing turns, pairs do not mix but for 0 x inf
    pos[25] = 77
    cache = empty_cache(5, page, hk, d)
    before = [c.clone() for c in cache]
    write((Q, K, V), pos, slots, freq, cache)
    turned, size = plain_rope(K, pos, freq, P.PIFA_ROPE_HALF)
    size = size.nan_to_num(0.0, 0.0, 0.0)
    check_store(before[0], cache[0], before[2], cache[2], turned, size, slots, page)
    check_store(before[1], cache[1], before[3], cache[3], V.double(), torch.zeros_like(size), slots, page)


@pytest.mark.parametrize("dtype,top,low", [(torch.bfloat16, 3.38e38, 1e-38), (torch.float16, 65504.0, 6e-8), (torch.bfloat16, 448.0, 0.0),
                                           (torch.bfloat16, 450.0, 2.0 ** -133)])
def test_largest_and_smallest_values(dtype, top, low):
    """Blocks of nothing but zeros, of the type's largest and smallest numbers, and of both."""
    hk, d, page, T = 3, 64, 16, 48
    K = torch.zeros((T, hk, d), dtype=dtype, device=DEV)
    K[:16, 1], K[16:32, 1], K[32:, 1] = top, low, low
    K[40, 1] = -top
    K[5:9, 2] = low
    slots, pos, freq = torch.arange(T, device=DEV), i32([0] * T), P.pifa_rope_frequencies(d, device=DEV)
    cache = empty_cache(3, page, hk, d)
    before = [c.clone() for c in cache]
    write((K, K, K), pos, slots, freq, cache)
    zero = torch.zeros(K.shape, dtype=torch.float64, device=DEV)
    for i in (0, 1):
        check_store(before[i], cache[i], before[2 + i], cache[2 + i], K.double(), zero, slots, page)
    assert (cache[3].view(U8)[:, :, 0] == 1).all() and (cache[1][:, :, 0].double() == 0).all()
    got, _ = P.pifa_cache_read_q8(*cache, slots, dtype=dtype)
    assert bool(got.isfinite().all())


def test_rows_of_a_block_in_any_order_and_a_token_rewritten():
    hk, d, page = 2, 128, 32
    g, freq = gen(8), P.pifa_rope_frequencies(d, device=DEV)
    cache = empty_cache(4, page, hk, d)
    first = torch.tensor([35, 33, 34, 32, 36, 47, 46, 70, 64, 65, 66, -1], device=DEV)   # gaps; block 4: 70 before its first token 64
    x = inputs(g, 12, 1, hk, d, torch.bfloat16)
    pos = i32(list(range(12)))
    for slots in (first, torch.tensor([40, 34, 33, -1], device=DEV), torch.tensor([67, 64, 71, 32], device=DEV)):
        y = [a[:len(slots)] * (1 if slots is first else 30) for a in x]
        before = [c.clone() for c in cache]
        write(y, pos[:len(slots)], slots, freq, cache)
        turned, size = plain_rope(y[1], pos[:len(slots)], freq, P.PIFA_ROPE_HALF)
        check_store(before[0], cache[0], before[2], cache[2], turned, size, slots, page)
        check_store(before[1], cache[1], before[3], cache[3], y[2].double(), torch.zeros_like(size), slots, page)


def test_a_scale_of_nan_stays_and_a_fresh_block_ignores_it():
    hk, d, page = 1, 64, 16
    freq, one = P.pifa_rope_frequencies(d, device=DEV), torch.ones((1, 1, d), dtype=torch.bfloat16, device=DEV)
    cache = empty_cache(2, page, hk, d)
    write((one, one, one), i32([0]), torch.tensor([3], device=DEV), freq, cache)      # tokens 0 to 2 were never written
    assert (cache[2].view(U8) == 0xff).all() and P.pifa_cache_read_q8(*cache, torch.tensor([3], device=DEV))[0].isnan().all()
    write((one, one, one), i32([0]), torch.tensor([0], device=DEV), freq, cache)
    K, V = P.pifa_cache_read_q8(*cache, torch.tensor([0], device=DEV))
    assert torch.equal(K, one) and torch.equal(V, one)
    assert (cache[2].view(U8)[1:] == 0xff).all() and (cache[0].view(U8)[1:] == 0x7f).all()


def test_slots_outside_the_cache_and_twice():
    hk, d, page, pages = 2, 64, 16, 3
    freq, one = P.pifa_rope_frequencies(d, device=DEV), torch.ones((5, 2, d), dtype=torch.bfloat16, device=DEV)
    room = empty_cache(pages + 2, page, hk, d, byte=0)
    inner = [c[1:-1] for c in room]
    slots = torch.tensor([0, pages * page, -2, 2 ** 40, pages * page - 16], device=DEV)
    write((one, one, one), i32([0] * 5), slots, freq, inner)
    assert P.pifa_device_status() == P.PIFA_ERR_DEVICE_INDEX
    for i in (0, 1):
        assert int((room[i].view(U8) != 0).sum()) == 2 * hk * d
        assert (inner[i][0, 0].double() == 256).all() and (inner[i][-1, 0].double() == 256).all()
        assert int((room[2 + i].view(U8) != 0xff).sum()) == 2 * hk
    for twice in ([5, 5], [16, 17, 18, 17], [3] * 5):
        write([one[:len(twice)]] * 3, i32([0] * len(twice)), torch.tensor(twice, device=DEV), freq, inner)
        assert P.pifa_device_status() == P.PIFA_ERR_DEVICE_INDEX
    many = torch.ones((50, 2, d), dtype=torch.bfloat16, device=DEV)
    write((many, many, many), i32([0] * 50), torch.full((50,), 32, device=DEV), freq, inner)
    assert P.pifa_device_status() == P.PIFA_ERR_DEVICE_INDEX
    for i in (0, 1):                                             # nothing outside the inner pages
        assert (room[i].view(U8)[0] == 0).all() and (room[i].view(U8)[-1] == 0).all()
        assert (room[2 + i].view(U8)[0] == 0xff).all() and (room[2 + i].view(U8)[-1] == 0xff).all()


# ---- reading back ------------------------------------------------------------------------------------------
def random_cache(g, pages, page, hk, d, heads_first=False, lo=97, hi=147):
    cache = empty_cache(pages, page, hk, d, heads_first)
    for c in cache[:2]:
        c.view(U8).copy_(torch.randint(0, 256, c.shape, device=DEV, generator=g).to(U8))
    for s in cache[2:]:
        s.view(U8).copy_(torch.randint(lo, hi, s.shape, device=DEV, generator=g).to(U8))
    return cache


@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,hk,d,page", [(1, 1, 64, 16), (301, 8, 128, 48), (33, 3, 96, 128), (5000, 2, 512, 16), (70000, 1, 16, 64)])
def test_read(T, hk, d, page, dtype, heads_first):
    g = gen(T)
    cache = random_cache(g, 40, page, hk, d, heads_first, 120 if dtype is torch.float16 else 12, 130 if dtype is torch.float16 else 245)
    slots = torch.randint(0, 40 * page, (T,), device=DEV, generator=g)     # in any order, some twice
    slots[T // 2:][:T // 3] = -1
    room = torch.full((T + 2, 2 * hk * d + 24), 9.0, dtype=dtype, device=DEV)
    K, V = (room[1:-1, 8 + i * (hk * d + 8):][:, :hk * d].unflatten(1, (hk, d)) for i in (0, 1))
    P.pifa_cache_read_q8(*cache, slots, K=K, V=V)
    kept = slots >= 0
    for got, i in ((K, 0), (V, 1)):
        at = slots[kept]
        want = values(cache[i], cache[2 + i])[at // page, at % page]
        assert torch.equal(got[kept].double().isnan(), want.isnan())
        err = (got[kept].double() - want).abs().nan_to_num(0.0)
        if dtype is torch.bfloat16:
            assert float(err.max()) == 0.0
        else:
            assert bool((err <= 2.0 ** -11 * want.abs().nan_to_num(0.0) + 2.0 ** -25).all())
        assert (got[~kept] == 9.0).all()
    assert (room[0] == 9).all() and (room[-1] == 9).all() and (room[:, :8] == 9).all() and (room[:, 8 + hk * d:16 + hk * d] == 9).all()
    K2, V2 = P.pifa_cache_read_q8(*cache, slots, dtype=dtype)
    assert K2.dtype is dtype and torch.equal(K2[kept].nan_to_num(0.5), K[kept].nan_to_num(0.5)) and (K2[~kept] == 0).all() and (V2[~kept] == 0).all()


def test_read_extreme_scales_and_slots():
    hk, d, page = 1, 16, 16
    cache = random_cache(gen(3), 4, page, hk, d)
    cache[0].view(U8)[:] = 0x7e                                  # 448
    cache[2].view(U8).copy_(torch.tensor([[[0]], [[255]], [[254]], [[135]]], dtype=U8))
    slots = torch.tensor([0, 16, 32, 48, 64, -7, -1], device=DEV)
    K, _ = P.pifa_cache_read_q8(*cache, slots)
    assert P.pifa_device_status() == P.PIFA_ERR_DEVICE_INDEX
    assert (K[0].double() == 448.0 * 2.0 ** -127).all() and K[1].isnan().all() and (K[2] == torch.finfo(torch.bfloat16).max).all()
    assert (K[3].double() == 448.0 * 256).all() and (K[4:] == 0).all()
    K, _ = P.pifa_cache_read_q8(*cache, slots[3:4], dtype=torch.float16)
    assert (K == 65504).all()


@pytest.mark.parametrize("new", [1, 70])
def test_offsets_past_32_bits(new):
    """A cache of 6 GiB a buffer: written, read and attended to at both ends."""
    hk, d, page, L = 2, 128, 64, 640
    pages = 6 * 2 ** 30 // (page * hk * d)
    cache = [torch.empty((pages, page, hk, d), dtype=U8, device=DEV).view(E4M3) for _ in range(2)]
    cache += [torch.empty((pages, 4, hk), dtype=U8, device=DEV).view(E8M0) for _ in range(2)]
    table = i32([[pages - 1, 0, pages - 3, 1, pages - 2, pages - 9, 5, pages - 8, 7, pages - 4]])
    pos = torch.arange(L, device=DEV)
    slots = table[0].long()[pos // page] * page + pos % page
    g, freq = gen(4), P.pifa_rope_frequencies(d, device=DEV)
    Q, K, V = inputs(g, L, 4, hk, d, torch.bfloat16)
    Qr = write((Q, K, V), pos.int(), slots, freq, cache)
    K8, V8 = P.pifa_cache_read_q8(*cache, slots)
    turned, size = plain_rope(K, pos.int(), freq, P.PIFA_ROPE_HALF)
    for got, want, extra in ((K8, turned, size), (V8, V.double(), 0 * size)):
        s = torch.exp2(torch.ceil(torch.log2(want.abs().view(L // 16, 16, hk, d).amax((1, 3)) / 448.0 * (1 + 1e-5)))).repeat_interleave(16, 0)[..., None]
        assert bool(((got.double() - want).abs() <= torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * s) + 1e-6 * extra).all())
    O = P.pifa_paged_attention_q8(Qr[L - new:], *cache, table, i32([0, new]), i32([L]), new)
    small = dict(Q=Qr[L - new:], k_cache=K8.view(L // page, page, hk, d), v_cache=V8.view(L // page, page, hk, d),
                 table=torch.arange(L // page, device=DEV, dtype=torch.int32)[None], q_start=i32([0, new]), kv_len=i32([L]))
    check_attention(small, O, d ** -0.5)


# ---- attention ---------------------------------------------------------------------------------------------
def make_q8(seed, lens, news, hq, hk, d, page, dtype, heads_first=False, spread=0, dead=0x7f, dead_scale=0xff):
    """Requests over shuffled pages of a quantised cache; blocks' scales spread over 2^+-spread; `dead` bytes wherever no request
    owns a token (or a block)."""
    a = make_attention(seed, lens, news, hq, hk, d, page, dtype, dead=math.nan)
    pages = a["k_cache"].shape[0]
    cache, g = empty_cache(pages, page, hk, d, heads_first, byte=dead), gen(seed + 1)
    for i, name in ((0, "k_cache"), (1, "v_cache")):
        x = a[name].double().view(pages, page // 16, 16, hk, d)
        if spread:
            x = x * torch.exp2(torch.randint(-spread, spread + 1, (pages, page // 16, 1, hk, 1), device=DEV, generator=g).double())
        most = x.abs().nan_to_num(0.0).amax((2, 4))
        e = torch.ceil(torch.log2(most.clamp(min=1e-30) / 448.0) - 1e-9)
        q = (x * torch.exp2(-e)[:, :, None, :, None]).float().clamp(-448, 448).to(E4M3).view(U8).view(pages, page, hk, d)
        gone = x.isnan().view(pages, page, hk, d)
        cache[i].view(U8).copy_(torch.where(gone, dead, q))
        some = ~x.isnan().all(2).all(-1)
        cache[2 + i].view(U8).copy_(torch.where(some, e + 127, dead_scale).to(U8))
    a.update(zip(("k8", "v8", "ks", "vs"), cache))
    a["k_cache"], a["v_cache"] = values(cache[0], cache[2]), values(cache[1], cache[3])   # what attention sees
    return a


def sizes(a, max_q):
    B, cols = a["table"].shape
    pages, page, hk, d = a["k8"].shape
    return a["Q"].shape[0], a["Q"].shape[1], hk, d, B, max_q, cols, page


def attend(a, max_q=None, scale=None, room=True, **kw):
    """room: for the keys and values of long chunks in 16 bits, if the call has a use for it."""
    if max_q is None:
        max_q = max([1] + (a["q_start"][1:] - a["q_start"][:-1]).tolist())
    size = sizes(a, max_q)
    need, most = P.pifa_paged_attention_workspace_size(*size[:6]), P.pifa_paged_attention_q8_workspace_size(*size)
    a["wide"] = room and most > need
    if not room:
        kw["workspace_tensor"] = torch.empty(need + 256, dtype=U8, device=DEV)
    return P.pifa_paged_attention_q8(a["Q"], a["k8"], a["v8"], a["ks"], a["vs"], a["table"], a["q_start"], a["kv_len"], max_q,
                                     scale=scale, **kw)


def check_attention(a, O, scale, slack=0.0):
    want, size, keys = plain_attention(a, scale)
    most = a["v_cache"].double().nan_to_num(0.0, 0.0, 0.0)
    most = float(most[a["table"].clamp(min=0).long().unique()].abs().max())
    w = U[O.dtype] if a.get("wide") else 2.0 ** -11
    tol = U[O.dtype] * want.abs() + (1.1 * w + 2e-4 + slack) * size + 2.0 ** -24 * (1.0 + keys) * most
    err = (O.double() - want).abs()
    assert bool((err <= tol).all()), (float((err - tol).max()), int((err > tol).sum()), (err > tol).nonzero()[:4].tolist())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", list(SHAPES))
def test_attention(name, dtype):
    lens, news, hq, hk, d, page = SHAPES[name]
    a = make_q8(len(name), lens, news, hq, hk, d, page, dtype)
    for room in (False, True):
        O = torch.full_like(a["Q"], math.nan)
        attend(a, O=O, room=room)
        check_attention(a, O, d ** -0.5)
        assert torch.equal(attend(a, room=room), O)     # and whatever order blocks run in
        if not a["wide"] and room:
            assert torch.equal(O, last)
        last = O


def test_long_chunks_take_the_room():
    """Which of the shapes above are brought to 16 bits first: those with more than 768 rows of a head."""
    for name, (lens, news, hq, hk, d, page) in SHAPES.items():
        cols = max(-(-n // page) for n in lens + [1]) + 1
        size = (sum(news), hq, hk, d, len(lens), max(news + [1]), cols, page)
        wide = P.pifa_paged_attention_q8_workspace_size(*size) > P.pifa_paged_attention_workspace_size(*size[:6])
        assert wide == (max(news) * hq // hk > 768), name
    assert P.pifa_paged_attention_q8_workspace_size(2048, 64, 8, 128, 200, 2048, 1000, 64) == P.pifa_paged_attention_workspace_size(
        2048, 64, 8, 128, 200, 2048)                    # 200 requests of up to 64000 tokens: more than a gigabyte


@pytest.mark.parametrize("name", ["decode_ragged_gqa", "few_tokens", "mixed", "prompt_1000_gqa", "chunk_group_3"])
def test_attention_scales_far_apart(name):
    """Keys and values whose blocks differ by up to 2^20 in size."""
    lens, news, hq, hk, d, page = SHAPES[name]
    a = make_q8(3, lens, news, hq, hk, d, page, torch.bfloat16, spread=5)
    a["Q"] = (a["Q"].float() / 32).to(torch.bfloat16)
    check_attention(a, attend(a, room=False), d ** -0.5)
    check_attention(a, attend(a), d ** -0.5)
    a = make_q8(4, lens, news, hq, hk, d, page, torch.bfloat16, spread=10)
    a["Q"] = (a["Q"].float() / 1024).to(torch.bfloat16)
    check_attention(a, attend(a, room=False), d ** -0.5)
    check_attention(a, attend(a), d ** -0.5)


@pytest.mark.parametrize("order", ["up", "down", "mixed"])
@pytest.mark.parametrize("new", [1, 5, 150, 400])
def test_attention_blocks_of_zeros_and_of_any_size(new, order):
    """Values whose blocks are nothing but zeros (the smallest scale) or differ by 2^120 in size: each key / value head against its own
    largest value, the weights' sum with all keys in it."""
    L, hq, hk, d, page = 900, 8, 4, 128, 32
    a = make_q8(17, [L], [new], hq, hk, d, page, torch.bfloat16)
    pages, g = a["table"][0, :-(-L // page)].long(), gen(18)
    blocks = len(pages) * page // 16
    size = torch.tensor([1, 1, 60, 100, 121, 160, 180], device=DEV)[torch.randint(0, 7, (blocks, hk), device=DEV, generator=g)]
    size[:, 0] = torch.where(torch.arange(blocks, device=DEV) % 3 > 0, 1, 121)       # a head whose values are mostly zeros
    if order != "mixed":
        size[:, 1:] = size[:, 1:].sort(0, descending=order == "down").values
    vs, v8 = a["vs"].view(U8), a["v8"].view(U8)
    vs[pages] = size.to(U8).view(len(pages), page // 16, hk)
    v8[pages] = torch.where(size.view(len(pages), page // 16, 1, hk, 1) == 1, 0, v8[pages].view(len(pages), page // 16, 16, hk, d)).view(len(pages), page, hk, d).to(U8)
    a["v_cache"] = values(a["v8"], a["vs"])
    want, s, keys = plain_attention(a, d ** -0.5)
    most = a["v_cache"][pages].flatten(0, 1)[:L].abs().amax((0, 2)).repeat_interleave(hq // hk)[None, :, None]
    for room in (False, True):
        O = attend(a, room=room)
        w = U[O.dtype] if a["wide"] else 2.0 ** -11
        err = (O.double() - want).abs()
        tol = U[O.dtype] * want.abs() + (1.1 * w + 2e-4) * s + 2.0 ** -24 * (1.0 + keys) * most
        assert bool((err <= tol).all()), (float((err - tol).max()), (err > tol).nonzero()[:4].tolist())


@pytest.mark.parametrize("size", [1e-30, 3e-5, 2e4, 1e30])
@pytest.mark.parametrize("name", ["decode_ragged_gqa", "prompt_1000_gqa"])
def test_attention_queries_of_any_size(name, size):
    """bf16 queries far outside fp16's range, of other sizes in other rows, and rows of zeros; the scale makes up for their size."""
    lens, news, hq, hk, d, page = SHAPES[name]
    a = make_q8(5, lens, news, hq, hk, d, page, torch.bfloat16)
    rows = torch.exp2(torch.arange(a["Q"].shape[0], device=DEV) % 3 - 1.0)[:, None, None]
    a["Q"] = (a["Q"].float() * size * rows).to(torch.bfloat16)
    a["Q"][0, 1] = 0.0
    for room in (False, True):
        check_attention(a, attend(a, scale=d ** -0.5 / size, room=room), d ** -0.5 / size)


@pytest.mark.parametrize("scale,size", [(1.0, 30.0), (-0.3, 2.0), (0.0, 1.0), (1e-3, 300.0)])
@pytest.mark.parametrize("name", ["decode_ragged_gqa", "prompt_1000_gqa"])
def test_attention_scores_of_any_size(name, scale, size):
    """Scores in the hundreds (one key takes all), negative scales, equal scores. Scores of size S carry fp32 errors of
    2^-23 S sqrt(d) or so, within 1e-3 of a weight here."""
    lens, news, hq, hk, d, page = SHAPES[name]
    a = make_q8(6, lens, news, hq, hk, d, page, torch.bfloat16)
    a["Q"] = (a["Q"].float() * size / 1.5).to(torch.bfloat16)
    for room in (False, True):
        check_attention(a, attend(a, scale=scale, room=room), scale, slack=2e-3)


@pytest.mark.parametrize("name", ["tokens_at_page_ends", "few_tokens_gqa", "mixed", "prompt_1000_gqa"])
def test_attention_bound_on_new_tokens_may_be_loose(name):
    lens, news, hq, hk, d, page = SHAPES[name]
    a = make_q8(5, lens, news, hq, hk, d, page, torch.bfloat16)
    for loose in (16, 100, 5000):
        if loose >= max(news):
            for room in (False, True):
                check_attention(a, attend(a, max_q=loose, room=room), d ** -0.5)


@pytest.mark.parametrize("room", [False, True])
@pytest.mark.parametrize("name", ["one_token", "few_tokens", "chunk_in_context", "mixed"])
def test_attention_strides_and_guards(name, room):
    lens, news, hq, hk, d, page = SHAPES[name]
    a = make_q8(9, lens, news, hq, hk, d, page, torch.bfloat16, heads_first=True)
    T = a["Q"].shape[0]
    wide = torch.full((T + 3, hq + 5, d), 3.0, dtype=torch.bfloat16, device=DEV)
    wide[:T, 2:2 + hq] = a["Q"]
    a["Q"] = wide[:, 2:2 + hq]
    frame = torch.full((T + 5, hq * d + 40), 9.0, dtype=torch.bfloat16, device=DEV)
    O = frame[1:-1, 16:16 + hq * d].unflatten(1, (hq, d))
    attend(a, O=O, room=room)
    a["Q"] = a["Q"][:T]
    check_attention(a, O[:T], d ** -0.5)
    assert (frame[0] == 9).all() and (frame[T + 1:] == 9).all() and (frame[:, :16] == 9).all() and (frame[:, 16 + hq * d:] == 9).all()


@pytest.mark.parametrize("dead,dead_scale", [(0x7f, 0xff), (0xff, 0xff), (0x7e, 0xfe), (0x55, 0), (0x7f, 127)])
@pytest.mark.parametrize("name", ["tokens_at_page_ends", "few_tokens", "mixed"])
def test_attention_ignores_what_no_request_owns(name, dead, dead_scale):
    lens, news, hq, hk, d, page = SHAPES[name]
    for dtype in DTYPES:
        a = make_q8(2, lens, news, hq, hk, d, page, dtype, dead=dead, dead_scale=dead_scale)
        b = make_q8(2, lens, news, hq, hk, d, page, dtype, dead=0, dead_scale=127)
        for room in (False, True):
            assert torch.equal(attend(a, room=room), attend(b, room=room))


@pytest.mark.parametrize("new", [1, 40, 400])
@pytest.mark.parametrize("what", ["k8", "ks", "vs"])
def test_attention_nan_stays_with_the_tokens_that_see_it(what, new):
    """A NaN key, or a scale of NaN: NaN for the rows that see (a token of) it, nothing for the others."""
    L, hq, hk, d, page = 260 + new, 4, 2, 128, 32
    a = make_q8(13, [L, 90], [new, 1], hq, hk, d, page, torch.bfloat16)
    good = attend(a)
    at = L - 20 if new > 1 else 100
    p, o = int(a["table"][0, at // page]), at % page
    if what == "k8":
        a[what].view(U8)[p, o, 1, 3] = 0x7f
    else:
        a[what].view(U8)[p, o // 16, 1] = 0xff
        at = at // 16 * 16
    O = attend(a)
    first = max(0, at - (L - new))                 # the first new token that sees key `at`
    assert bool(O[first:new, 2:].isnan().all())
    assert torch.equal(O[:new, :2], good[:new, :2]) and torch.equal(O[new:], good[new:])
    if what != "vs":
        assert torch.equal(O[:first], good[:first])


def test_attention_reports_bad_tables_and_bounds():
    for new in (400, 1, 40):
        a = make_q8(7, [200 + new, 90], [new, 1], 4, 2, 128, 16, torch.bfloat16)
        good = attend(a)
        for bad in (-1, 10 ** 6, 2 ** 31 - 1):
            b = dict(a, table=a["table"].clone())
            b["table"][0, 3] = bad
            O = attend(b)
            assert P.pifa_device_status() == P.PIFA_ERR_DEVICE_INDEX
            assert torch.equal(O[new:], good[new:])
            z = dict(a, k_cache=a["k_cache"].clone(), v_cache=a["v_cache"].clone(), wide=b["wide"])
            z["k_cache"][int(a["table"][0, 3])] = 0.0
            z["v_cache"][int(a["table"][0, 3])] = 0.0
            check_attention(z, O, 128 ** -0.5)
        b = dict(a, kv_len=i32([10 ** 6, 90]))
        for room in (False, True):
            O = attend(b, room=room)
            assert P.pifa_device_status() in (P.PIFA_ERR_CAPACITY, P.PIFA_ERR_DEVICE_INDEX)
            check_attention(a, torch.cat([good[:new], O[new:]]), 128 ** -0.5)
        O = torch.full_like(a["Q"], 5.0)
        attend(dict(a, q_start=i32([0, new + 1, new])), max_q=new + 1, O=O)
        assert P.pifa_device_status() == P.PIFA_ERR_DEVICE_INDEX and (O == 5.0).all()
    O = torch.full_like(a["Q"], 5.0)
    attend(a, max_q=3, O=O)
    assert P.pifa_device_status() == P.PIFA_ERR_CAPACITY
    assert (O[3:40] == 5.0).all()
    check_attention(a, torch.cat([O[:3], good[3:40], O[40:]]), 128 ** -0.5)


def test_attention_on_two_streams_at_once():
    hq, hk, d, page = 16, 4, 128, 32
    sets = [make_q8(21, [3000, 40, 700], [300, 1, 77], hq, hk, d, page, torch.bfloat16),
            make_q8(22, [9000, 5000], [1, 1], hq, hk, d, page, torch.bfloat16),
            make_q8(23, [6000], [70], hq, hk, d, page, torch.float16),
            make_q8(24, [200] * 40, [3] * 40, hq, hk, d, page, torch.bfloat16)]
    serial = [attend(a) for a in sets]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    bounds = [300, 1, 70, 3]
    for k in range(24):
        for s in (0, 1):
            with torch.cuda.stream(streams[s]):
                i = (k + 2 * s) % 4
                got[s].append((i, attend(sets[i], max_q=bounds[i])))
    torch.cuda.synchronize()
    for s in (0, 1):
        for i, O in got[s]:
            assert torch.equal(O, serial[i])


# ---- together ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_serving_loop(dtype):
    """Page tables, the write and the attention of prompts, then decode steps replayed from one graph, against 64 bits on
    what the cache holds, and the cache against the tokens that went in."""
    B, hq, hk, d, page, steps_, cols = 5, 8, 2, 128, 32, 20, 8
    g = gen(77)
    cache, freq = empty_cache(B * cols + 2, page, hk, d), P.pifa_rope_frequencies(d, device=DEV)
    free = torch.randperm(B * cols + 2, device=DEV, generator=g).int()
    head, lens, table = i32([0]), i32([0] * B), torch.full((B, cols), -1, dtype=torch.int32, device=DEV)
    prompt = [3, 16, 47, 96, 230 if dtype is torch.float16 else 130]
    sent = [[] for _ in range(B)]

    def step(x, new, T, max_q, out, Qr, O):
        start, kv, pos, slots, _ = P.pifa_page_tables(lens, new, page, free, head, table, T, out=out)
        Q, K, V = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        P.pifa_rope_cache_q8(Q, K, V, pos, slots, freq, *cache, Qr=Qr)
        return P.pifa_paged_attention_q8(Qr, *cache, table, start, kv, max_q, O=O)

    def buffers(T):
        return ((torch.empty(B + 1, dtype=torch.int32, device=DEV), lens, torch.empty(T, dtype=torch.int32, device=DEV),
                 torch.empty(T, dtype=torch.int64, device=DEV), head),
                torch.empty((T, hq, d), dtype=dtype, device=DEV), torch.zeros((T, hq, d), dtype=dtype, device=DEV))

    def check(out, Qr, O, max_q):
        n = int(out[0][-1])
        a = dict(Q=Qr[:n], k_cache=values(cache[0], cache[2]), v_cache=values(cache[1], cache[3]), table=table, q_start=out[0], kv_len=lens,
                 wide=max_q * hq // hk > 768)
        check_attention(a, O[:n], d ** -0.5)

    T = sum(prompt) + 4                                          # padded
    x = torch.randn((T, hq + 2 * hk, d), device=DEV, generator=g).to(dtype)
    buf = buffers(T)
    step(x, i32(prompt), T, max(prompt), *buf)
    check(*buf, max(prompt))
    at = 0
    for b, n in enumerate(prompt):
        sent[b] += list(x[at:at + n, hq + hk:])
        at += n
    ones, x1, buf = i32([1] * B), torch.empty((B, hq + 2 * hk, d), dtype=dtype, device=DEV), buffers(B)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(x1, ones, B, 1, *buf)
    for k in range(steps_):
        x1.copy_(torch.randn(x1.shape, device=DEV, generator=g) * (1 + k % 5))
        graph.replay()
        torch.cuda.synchronize()
        if k % 6 == 5:
            check(*buf, 1)
        for b in range(B):
            sent[b].append(x1[b, hq + hk:].clone())
    for b in range(B):                                           # values are not turned: what went in, within the roundings
        n = int(lens[b])
        assert n == prompt[b] + steps_
        t = torch.arange(n, device=DEV)
        _, V = P.pifa_cache_read_q8(*cache, table[b].long()[t // page] * page + t % page, dtype=dtype)
        want = torch.stack(sent[b]).double()
        s = cache[3].double()[table[b].long()[t // page], t % page // 16][..., None]
        # half a step, and up to four risings of the scale, each half a step of the subnormal range
        assert bool(((V.double() - want).abs() <= torch.maximum(2.0 ** -4 * want.abs(), 5 * 2.0 ** -10 * s)).all())
