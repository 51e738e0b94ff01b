"""Attention over a cache in 8 bits where one key has nearly all the weight and a value of zero, and the output is what is left to the
others: thousands of small weights, which have to be in the sum of the values as they are in the sum of the weights.

Bounds, first order: the output is rounded once, u |o|; a weight is rounded to w (fp16; dtype where the cache was brought to 16 bits
before), 10% over; 2e-4 for fp32 scores, exponentials and sums. fp16 weights are held 2^7 times as large as against the largest,
so that one below fp16's normal range is off by 2^-25 2^-7 of the largest at most, and the sum of weights is the largest at least:
2^-32 max |v| a key. bf16 has no such range. An output in fp16 below its normal range is off by 2^-25.
"""
import pytest
import torch

from paper_2501_19090_gb300 import pifa as P
from test_attention_path_gpu import gen, plain_attention
from test_cache_q8_gpu import DTYPES, E4M3, U, U8, attend, make_q8, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HQ, HK, PAGE = 16, 2, 64        # groups of 8: a new token has 8 rows, two 16, and so on
# new tokens of a request, alike requests (enough of them that most of a head's keys are added up in one piece), room for 16 bits
PATHS = {"rows_8": (1, 600, False), "rows_16": (2, 600, False), "chunk": (60, 80, False), "long_chunk": (150, 32, False),
         "long_chunk_widened": (150, 32, True)}
L = 4000


def sink(n, d, dtype, nats, sink_scale=127):
    """A request whose key 0 scores `nats` above the others' mean, which are normal with a deviation of about a half."""
    a, g = make_q8(L + n, [L], [n], HQ, HK, d, PAGE, dtype), gen(d + n)
    pages = a["table"][0, :-(-L // PAGE)].long()
    k = torch.randn((len(pages), PAGE, HK, d), device=DEV, generator=g)
    v = torch.randn(k.shape, device=DEV, generator=g).abs() + 0.5
    k[..., 0] = 0.0
    k[0, 0, :, 0] = 16.0
    v[0, 0] = 0.0
    for name, x in (("k8", k), ("v8", v)):
        a[name].view(U8)[pages] = x.to(E4M3).view(U8)
    for name in ("ks", "vs"):
        a[name].view(U8)[pages] = 127
    a["vs"].view(U8)[pages[0], 0] = sink_scale
    a["Q"] = (torch.randn(a["Q"].shape, device=DEV, generator=g) * 0.5).to(dtype)
    a["Q"][..., 0] = nats * d ** 0.5 / 16.0
    a["k_cache"], a["v_cache"] = values(a["k8"], a["ks"]), values(a["v8"], a["vs"])
    return a, float(v.max())


def check(a, path, slack, scale=None):
    """The request, many times over the same pages, each against 64 bits."""
    n, B, room = PATHS[path]
    dtype, d = a["Q"].dtype, a["Q"].shape[2]
    many = dict(a, Q=a["Q"].repeat(B, 1, 1), table=a["table"].repeat(B, 1), kv_len=a["kv_len"].repeat(B),
                q_start=torch.arange(B + 1, device=DEV, dtype=torch.int32) * n)
    O = attend(many, max_q=n, room=room, scale=scale)
    assert P.pifa_device_status() == P.PIFA_OK and many["wide"] == (path == "long_chunk_widened")
    want, size, _ = plain_attention(a, d ** -0.5 if scale is None else scale)
    w = U[dtype] if many["wide"] else 2.0 ** -11
    tol = U[dtype] * want.abs() + (1.1 * w + 2e-4) * size
    if not (many["wide"] and dtype is torch.bfloat16):
        tol += slack
    if dtype is torch.float16:
        tol += 2.0 ** -25
    err = (O.double().view(B, n, HQ, d) - want).abs()
    assert bool((err <= tol).all()), (float((err / want.abs()).max()), float((tol / want.abs()).min()), int((err > tol).sum()))
    return want


@pytest.mark.parametrize("nats", [4, 14, 18, 20])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("path", list(PATHS))
def test_many_small_weights_beside_a_large_one(path, dtype, d, nats):
    for sink_scale in (127, 100):
        a, most = sink(PATHS[path][0], d, dtype, nats, sink_scale)
        assert float(check(a, path, 2.0 ** -32 * L * most).min()) > 0.0


@pytest.mark.parametrize("scale", [0.0, 1e-44, 1e-37, 1e-20])
@pytest.mark.parametrize("path", list(PATHS))
def test_equal_weights(path, scale):
    """Scales so small that all weights are equal: what brings the reference 7 below the maximum must stay finite."""
    a, most = sink(PATHS[path][0], 64, torch.float16, 4)
    check(a, path, 2.0 ** -32 * L * most, scale)


@pytest.mark.parametrize("dtype,top", [(torch.bfloat16, 119), (torch.float16, 7)])
@pytest.mark.parametrize("new", [1, 2, 60, 150])
def test_values_near_the_largest_of_the_type(new, dtype, top):
    """One key takes all, and its values are the largest that a block holds: sums that are cut along the keys stay finite."""
    d = 128
    a, _ = sink(new, d, dtype, 60)
    page = int(a["table"][0, 0])
    a["v8"].view(U8)[page, 0] = torch.full((HK, d), 448.0, device=DEV).to(E4M3).view(U8)
    a["vs"].view(U8)[page, 0] = 127 + top
    a["k_cache"], a["v_cache"] = values(a["k8"], a["ks"]), values(a["v8"], a["vs"])
    want, _, _ = plain_attention(a, d ** -0.5)
    for room in (False, True):
        O = attend(a, room=room)                         # one request: its keys are cut
        err = (O.double() - want).abs()
        assert bool(O.isfinite().all()) and bool((err <= (U[dtype] + 1.1 * 2.0 ** -8 + 2e-4) * want).all()), float((err / want).max())


@pytest.mark.parametrize("path", list(PATHS))
def test_the_largest_weight_may_come_late_and_in_steps(path):
    """Maxima that rise by less than what raises the reference, so that weights reach the largest that they may: scores rise by 5 in
    the exponent from one part of the keys to the next, and fall again."""
    a, most = sink(PATHS[path][0], 128, torch.bfloat16, 18)
    pages = a["table"][0, :-(-L // PAGE)].long()
    for steps in ([0, 1, 2, 3, 4, 5, 4, 3, 2, 1], [0, 1.55, 0, 1.58, 0.5], [5, 0, 1]):
        part = torch.arange(len(pages), device=DEV) * len(steps) // len(pages)
        lift = torch.tensor(steps, device=DEV, dtype=torch.float32)[part][:, None, None]
        # the score of column 0 is nats / 16 of its key, 18 / 16 log2(e) in the exponent: 5 of them are 3.08 of the key
        a["k8"].view(U8)[pages, :, :, 0] = (lift * 3.08).expand(len(pages), PAGE, HK).to(E4M3).view(U8)
        a["k_cache"] = values(a["k8"], a["ks"])
        check(a, path, 2.0 ** -32 * L * most)
