"""Long requests whose keys are cut into many pieces: inputs that make every single piece visible in the output.

counts  equal scores, and key j's value is the unit vector of column (j / 16) mod head_dim: an output column is the number
        of its keys that the row sees over the number of all. The weights are 1, so products and sums are whole
        numbers below 2^24, exact in fp32; the reciprocal, its product and the rounding to the type leave u + 2^-22.
hot     one key of each key / value head has a score that is larger than the others' by 40 or more, so that all others
        together weigh 40000 e^-40 < 2e-13 of it: the output is that key's value, with the roundings of its weight
        and of the output: 2 u and 1 % for what is of second order.
The checks are themselves checked on the CPU: an oracle that leaves out, or takes twice, one piece of keys fails them."""
import pytest
import torch

from paper_2501_19090_gb300 import pifa as P

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
DTYPES = [torch.bfloat16, torch.float16]
# (kv lengths, new tokens, query heads, kv heads, head_dim, page)
SHAPES = {
    "decode_40000": ([40000], [1], 2, 1, 128, 256),
    "decode_16000_gqa": ([16000], [1], 64, 8, 128, 64),
    "decode_ragged_d64": ([9000, 1, 16000, 64, 3001, 500], [1] * 6, 8, 4, 64, 16),
    "four_tokens": ([12000, 40], [4, 4], 8, 4, 128, 32),
    "chunk_over_8000": ([8200], [200], 64, 8, 128, 64),
    "chunk_over_30000_d64": ([30040, 500], [40, 4], 8, 2, 64, 16),
    "chunk_few_items": ([6001], [70], 4, 2, 128, 32),
    "long_among_short": ([16000] + [500] * 7, [4] * 8, 64, 8, 128, 64),
}


def build(name, dtype, device, seed):
    """Requests over shuffled pages; the dense keys and values (requests' tokens in a row) still to be filled in."""
    lens, news, hq, hk, d, page = SHAPES[name]
    g = torch.Generator().manual_seed(seed)
    want = [-(-n // page) for n in lens]
    order = torch.randperm(sum(want), generator=g).to(torch.int32)
    table, at = torch.full((len(lens), max(want)), -1, dtype=torch.int32), 0
    for b, w in enumerate(want):
        table[b, :w] = order[at:at + w]
        at += w
    start = torch.tensor([0] + news).cumsum(0).to(torch.int32)
    Q = torch.randn((int(start[-1]), hq, d), generator=g).to(dtype)
    slots = torch.cat([table[b, :w].repeat_interleave(page)[:n].long() * page + torch.arange(n) % page
                       for b, (w, n) in enumerate(zip(want, lens))])
    return dict(Q=Q.to(device), table=table.to(device), q_start=start.to(device), kv_len=torch.tensor(lens, dtype=torch.int32, device=device),
                slots=slots.to(device), pages=sum(want), lens=lens, news=news, hk=hk, page=page, g=g)


def rows(a):
    """(request, index among its new tokens, keys that it sees) of each row of Q."""
    return [(b, i, L - n + i + 1) for b, (L, n) in enumerate(zip(a["lens"], a["news"])) for i in range(n)]


def shares(n, d, times=None):
    """Of n keys, the share of each column's, each key counted `times` times."""
    times = torch.ones(n, dtype=torch.float64) if times is None else times
    return torch.zeros(d, dtype=torch.float64).index_add_(0, torch.arange(n) // 16 % d, times) / times.sum()


def counts(name, dtype, device):
    """Inputs, and the exact outputs (T x heads x head_dim)."""
    a = build(name, dtype, device, 1)
    d = a["Q"].shape[2]
    a["Q"].zero_()
    j = torch.cat([torch.arange(n) for n in a["lens"]])
    V = torch.nn.functional.one_hot(j // 16 % d, d).to(dtype).to(device)[:, None].expand(-1, a["hk"], -1)
    K = torch.randn((len(j), a["hk"], d), generator=a["g"]).to(dtype).to(device)
    want = torch.stack([shares(n, d) for _, _, n in rows(a)])
    return a, K, V, want.to(device)[:, None].expand(-1, a["Q"].shape[1], -1)


def check_counts(got, want, dtype):
    return bool(((got.double() - want).abs() <= (U[dtype] + 2.0 ** -22) * want).all())


def hot(name, dtype, device, seed):
    """Inputs, the hot keys of each (request, kv head), and the outputs."""
    a = build(name, dtype, device, seed)
    T, hq, d = a["Q"].shape
    hk, G = a["hk"], hq // a["hk"]
    first = torch.tensor([0] + a["lens"]).cumsum(0)
    # one direction for all rows, so that a key of that direction has a score of 60 with each, and others none
    one = torch.zeros(d)
    one[::2] = 1.0
    a["Q"][:] = one.to(a["Q"])
    K = torch.zeros((int(first[-1]), hk, d), dtype=dtype)
    K[..., 1::2] = torch.randn((int(first[-1]), hk, d // 2), generator=a["g"]).to(dtype)
    V = torch.randn((int(first[-1]), hk, d), generator=a["g"]).to(dtype)
    keys = []
    for b, (L, n) in enumerate(zip(a["lens"], a["news"])):
        seen = L - n + 1                        # by every row
        places = [0, seen - 1] + [(seen * k // 61) // 16 * 16 - e for k in range(1, 61) for e in (0, 1)]
        pick = torch.randperm(len(places), generator=a["g"])
        keys.append([max(0, min(places[pick[(h + seed) % len(places)]], seen - 1)) for h in range(hk)])
        for h, k in enumerate(keys[-1]):
            K[first[b] + k, h, ::2] = 60.0 * d ** 0.5 / (d / 2)
    V, K = V.to(device), K.to(device)
    want = torch.empty((T, hq, d), dtype=torch.float64, device=device)
    for r, (b, _, _) in enumerate(rows(a)):
        for h in range(hk):
            want[r, h * G:(h + 1) * G] = V[first[b] + keys[b][h], h].double()
    return a, K, V, keys, want


def check_hot(got, want, dtype):
    return bool(((got.double() - want).abs() <= 2.02 * U[dtype] * want.abs() + 2e-12).all())


# ---- the checks ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("name", list(SHAPES))
def test_the_counts_show_a_piece_that_is_lost_or_taken_twice(name):
    (L, *_), (new, *_), _, _, d, _ = SHAPES[name]
    right = shares(L, d)                        # of the first request's last row
    for dtype in DTYPES:
        assert check_counts(right.to(dtype), right, dtype)
        for size in (64, 128):
            for k0 in range(0, L - new - size, L // 23):
                for factor in (0.0, 2.0):
                    times = torch.ones(L, dtype=torch.float64)
                    times[k0:k0 + size] = factor
                    assert not check_counts(shares(L, d, times).to(dtype), right, dtype)


def test_a_hot_key_outweighs_all_others():
    name, dtype = "four_tokens", torch.bfloat16
    a, K, V, keys, want = hot(name, dtype, "cpu", 3)
    d, G = K.shape[2], a["Q"].shape[1] // a["hk"]
    scale = d ** -0.5
    for keep in (True, False):      # an oracle with all keys, and one that loses the hot key's piece
        got = torch.empty_like(want)
        first = 0
        for b, L in enumerate(a["lens"]):
            for r, (rb, _, n) in enumerate(rows(a)):
                if rb != b:
                    continue
                for h in range(a["hk"]):
                    s = K[first:first + n, h].double() @ a["Q"][r, h * G].double() * scale
                    if not keep:
                        s[keys[b][h] // 64 * 64:keys[b][h] // 64 * 64 + 64] = -float("inf")
                        if s.max() == -float("inf"):
                            s[:] = 0.0
                    got[r, h * G:(h + 1) * G] = torch.softmax(s, 0) @ V[first:first + n, h].double()
            first += L
        assert check_hot(got.to(dtype), want, dtype) == keep


# ---- the kernels --------------------------------------------------------------------------------------------
def run(a, K, V, dtype):
    d, device = K.shape[2], K.device
    kc, vc = (torch.full((a["pages"] * a["page"], a["hk"], d), float("nan"), dtype=dtype, device=device) for _ in range(2))
    kc[a["slots"]], vc[a["slots"]] = K, V
    O = torch.full_like(a["Q"], float("nan"))
    P.pifa_paged_attention(a["Q"], kc.view(-1, a["page"], a["hk"], d), vc.view(-1, a["page"], a["hk"], d), a["table"], a["q_start"],
                           a["kv_len"], max(a["news"]), O=O)
    assert P.pifa_device_status() == P.PIFA_OK
    return O


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", list(SHAPES))
def test_every_piece_is_counted_once(name, dtype):
    a, K, V, want = counts(name, dtype, "cuda:0")
    got = run(a, K, V, dtype)
    assert check_counts(got, want, dtype), float(((got.double() - want).abs() / want.clamp(min=1e-9)).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", list(SHAPES))
def test_every_piece_can_hold_the_largest_score(name, dtype):
    for seed in range(12):
        a, K, V, keys, want = hot(name, dtype, "cuda:0", seed)
        got = run(a, K, V, dtype)
        assert check_hot(got, want, dtype), (seed, keys, ((got.double() - want).abs() > 2.02 * U[dtype] * want.abs()).sum().item())
