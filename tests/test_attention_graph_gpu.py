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
