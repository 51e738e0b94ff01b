"""Graphs captured with the binding's default scratch, replayed beside eager calls."""
import math

import pytest
import torch

from paper_2501_19090_gb300 import pifa as P
from test_attention_path_gpu import DEV, attend, check_attention, make_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("warm", [False, True])
@pytest.mark.parametrize("news,lens", [([1, 1, 1], [2000, 33, 64]), ([40, 1], [900, 300])])
def test_attention_graph_with_default_scratch(news, lens, warm):
    """Captured on a stream, then larger eager calls on it, then tensors over whatever they gave back: replays neither
    change those tensors nor are changed by them, also when an eager call runs beside the replay."""
    hq, hk, d, page = 8, 2, 128, 16
    a = make_attention(31, lens, news, hq, hk, d, page, torch.bfloat16)
    big = make_attention(32, [1500, 700], [900, 700], hq, hk, d, page, torch.bfloat16)
    want, big_want = attend(a), attend(big)
    O, big_O = torch.empty_like(a["Q"]), torch.empty_like(big["Q"])
    stream, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        if warm:
            attend(a, max_q=max(news), O=O)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            attend(a, max_q=max(news), O=O)
            attend(a, max_q=max(news), O=O)
        attend(big, max_q=900, O=big_O)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        fill = [torch.full((n,), 77, dtype=torch.uint8, device=DEV) for n in (2 ** 20, 2 ** 21, 2 ** 22, 2 ** 24, 2 ** 26) * 4]
    O.fill_(math.nan)
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(O, want)
    assert all(bool((x == 77).all()) for x in fill)
    for _ in range(20):          # a replay on one stream, an eager call on the stream of the capture
        with torch.cuda.stream(other):
            graph.replay()
        with torch.cuda.stream(stream):
            attend(big, max_q=900, O=big_O)
    torch.cuda.synchronize()
    assert torch.equal(O, want) and torch.equal(big_O, big_want)
    check_attention(a, O, d ** -0.5)
    assert P.pifa_device_status() == P.PIFA_OK


def small_layer(m, n, r, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    order = torch.randperm(m, device=DEV, generator=g)
    rand = lambda *shape: (torch.randn(shape, device=DEV, generator=g) * r ** -0.5).to(torch.bfloat16)
    return (rand(r, n), rand(m - r, r), order[:r].sort().values.int(), order[r:].sort().values.int()), rand


@pytest.mark.parametrize("what", ["forward", "grouped", "backward", "accumulate"])
def test_projections_graph_with_default_scratch(what):
    """As above for a captured projection, its gradient and the calibration's accumulators."""
    n, r = 1024, 512
    layer, rand = small_layer(n, n, r, 5)
    pair = [torch.cat([w, w]) for w in layer[:2]] + [torch.cat([i, i + n]) for i in layer[2:]]

    def call(T, X, dY, out):
        if what == "forward":
            out["Y"] = P.pifa_forward(X, *layer)
        elif what == "grouped":
            out["Y"] = P.pifa_forward_grouped(2, X, *pair)
        elif what == "backward":
            out.update(zip(("dX", "dWp", "dC"), P.pifa_backward(X, *layer, dY)))
        else:
            out["XXt"] = torch.zeros((n, n), device=DEV)
            P.pifa_m_accumulate(None, X, None, 0.5, out["XXt"])

    X, dY, big = rand(24, n), rand(24, n), rand(4096, n)
    want, got, rest = {}, {}, {}
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        call(24, X, dY, want)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            call(24, X, dY, got)
        call(4096, big, big, rest)
        torch.cuda.synchronize()
        fill = [torch.full((k,), 77, dtype=torch.uint8, device=DEV) for k in (2 ** 12, 2 ** 16, 2 ** 20, 2 ** 22, 2 ** 24) * 6]
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert set(got) == set(want) and all(torch.equal(got[k], want[k]) for k in want)
    assert all(bool((x == 77).all()) for x in fill)
    assert P.pifa_device_status() == P.PIFA_OK
