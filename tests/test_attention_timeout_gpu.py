"""Attention of chunks whose waits run out: with a bound of next to nothing the kernel's ordinary waits, for copies and products
of some microseconds, give up. The call ends, reports PIFA_ERR_TIMEOUT, writes nothing outside its outputs, and leaves the
next call as it would have been."""
import pytest
import torch

from paper_2501_19090_gb300 import pifa as P
from test_attention_path_gpu import check_attention, make_attention

pytestmark = pytest.mark.gpu

# (kv lengths, new tokens, query heads, kv heads, head_dim, page): items that are cut, whole ones, pages of every form
SHAPES = {"cut": ([8200], [200], 64, 8, 128, 64), "cut_d64": ([6001, 300], [70, 2], 8, 2, 64, 16), "prompt": ([2048], [2048], 8, 8, 128, 16),
          "ragged": ([900, 0, 64, 2500], [300, 4, 64, 1], 8, 4, 128, 256)}


@pytest.fixture(autouse=True)
def _bound():
    yield
    P.pifa_set_wait_timeout(0)
    P.pifa_device_status()


@pytest.mark.parametrize("name", list(SHAPES))
def test_waits_that_run_out(name):
    lens, news, hq, hk, d, page = SHAPES[name]
    a = make_attention(6, lens, news, hq, hk, d, page, torch.bfloat16)
    call = lambda O: P.pifa_paged_attention(a["Q"], a["k_cache"], a["v_cache"], a["table"], a["q_start"], a["kv_len"], max(news), O=O)
    T = a["Q"].shape[0]
    room = torch.full((T + 2, hq, d), 9.0, dtype=torch.bfloat16, device=a["Q"].device)
    want = call(torch.empty_like(a["Q"]))
    assert P.pifa_device_status() == P.PIFA_OK
    check_attention(a, want, d ** -0.5)
    for ns in (1, 1, 500, 2000, 5000, 10000, 20000):
        P.pifa_set_wait_timeout(ns)
        call(room[1:-1])
        status = P.pifa_device_status()
        assert status == P.PIFA_ERR_TIMEOUT or (ns > 1 and status == P.PIFA_OK)
        assert bool((room[0] == 9.0).all() and (room[-1] == 9.0).all())
        P.pifa_set_wait_timeout(0)
        O = call(torch.full_like(want, float("nan")))
        assert P.pifa_device_status() == P.PIFA_OK and torch.equal(O, want)
