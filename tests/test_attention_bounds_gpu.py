"""Attention over arrays that do not hold what the header asks for: what is latched, and that nothing is written
outside the call's buffers."""
import pytest
import torch

from paper_2501_19090_gb300 import pifa as P
from test_attention_path_gpu import DEV, check_attention, i32, make_attention

pytestmark = pytest.mark.gpu


def guarded(a, hq, hk, d, max_q):
    """(workspace of exactly the size asked for, the bytes around it)."""
    need = P.pifa_paged_attention_workspace_size(a["Q"].shape[0], hq, hk, d, a["kv_len"].numel(), max_q)
    room = torch.full((need + 3 * 2 ** 20,), 0x5a, dtype=torch.uint8, device=DEV)
    lead = 2 ** 20 - room.data_ptr() % 256
    return room[lead:lead + need], (room[:lead], room[lead + need:])


def attend(a, max_q, ws, O):
    return P.pifa_paged_attention(a["Q"], a["k_cache"], a["v_cache"], a["table"], a["q_start"], a["kv_len"], max_q, O=O,
                                  workspace_tensor=ws)


# T tokens, requests, query heads, kv heads, head_dim, bound on new tokens: the last one picks the kernel. With starts
# 0, T, 0, T, ... every second request has T tokens, so that 4096 requests have more items than any list has room for.
CASES = {"few_rows": (16, 6, 4, 4, 128, 16), "one_token": (3, 64, 8, 1, 64, 1), "chunk": (700, 2, 8, 2, 128, 700),
         "list": (8192, 64, 8, 1, 128, 8192), "workspace": (8192, 4096, 8, 1, 64, 8192)}


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("shape", ["in_turn", "one_step_back", "below_zero"])
def test_starts_that_are_not_ascending(name, shape):
    T, B, hq, hk, d, max_q = CASES[name]
    a = make_attention(3, [40] + [1] * (B - 1), [T] + [0] * (B - 1), hq, hk, d, 16, torch.bfloat16)
    good = a["q_start"]
    a["q_start"] = i32({"in_turn": [T * (b % 2) for b in range(B + 1)],
                        "one_step_back": [T] * B + [T - 1] if B > 2 else [0, T, T - 1],
                        "below_zero": [0, -5] + [T] * (B - 1)}[shape])
    ws, guards = guarded(a, hq, hk, d, max_q)
    O = torch.full_like(a["Q"], 5.0)
    attend(a, max_q, ws, O)
    assert P.pifa_device_status() in (P.PIFA_ERR_DEVICE_INDEX, P.PIFA_ERR_CAPACITY)
    assert bool((O == 5.0).all()) and all(bool((x == 0x5a).all()) for x in guards)
    a["q_start"] = good                      # and the next call is none the worse for it
    attend(a, T, None, O) if T > max_q else attend(a, max_q, ws, O)
    assert P.pifa_device_status() == P.PIFA_OK
    check_attention(a, O, d ** -0.5)


@pytest.mark.parametrize("max_q", [1, 300])
def test_no_request_has_a_token(max_q):
    a = make_attention(4, [40, 7, 300], [5, 2, 1], 4, 2, 128, 16, torch.bfloat16)
    a["q_start"] = i32([0, 0, 0, 0])
    ws, guards = guarded(a, 4, 2, 128, max_q)
    O = torch.full_like(a["Q"], 5.0)
    attend(a, max_q, ws, O)
    assert P.pifa_device_status() == P.PIFA_OK
    assert bool((O == 5.0).all()) and all(bool((x == 0x5a).all()) for x in guards)
