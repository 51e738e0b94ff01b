"""Page tables of steps that do not fit, and of no requests."""
import random

import pytest
import torch

from paper_2501_19090_gb300 import pifa as P
from test_attention_path_gpu import DEV, attend, check_attention, i32, make_attention, plain_tables, table_case

pytestmark = pytest.mark.gpu


def cut(new, T):
    """The tokens of each request that `T` rows have room for."""
    out = []
    for n in new:
        out.append(min(n, T - sum(out)))
    return out


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,page,share", [(3, 16, 0.6), (1, 16, 0.5), (5, 1, 0.3), (64, 16, 0.0), (64, 16, 0.97), (2500, 32, 0.4)])
def test_tokens_that_do_not_fit_are_no_part_of_the_step(B, page, share, in_place):
    """Requests keep the tokens that have rows: starts, lengths, pages and the free list's head agree on them."""
    rng = random.Random(B + int(100 * share))
    old, new, free, first, table = table_case(rng, B, page, 300, 40)
    new[0] += 2
    T = int(share * sum(new))
    want, start, kv, pos, slots, nxt = plain_tables(old, cut(new, T), page, free, first, [list(r) for r in table], T)
    lens, head, dev_table = i32(old), i32([first]), i32(table)
    empty = lambda n, dtype=torch.int32: torch.full((n,), -3, dtype=dtype, device=DEV)
    out = (empty(B + 1), lens if in_place else empty(B), empty(T), empty(T, torch.int64), head if in_place else empty(1))
    P.pifa_page_tables(lens, i32(new), page, i32(free), head, dev_table, T, out=out)
    assert P.pifa_device_status() == P.PIFA_ERR_CAPACITY
    assert [x.tolist() for x in out] == [start, kv, pos, slots, [nxt]]
    assert dev_table.tolist() == want


def test_attention_of_a_step_that_does_not_fit():
    """The tokens that fit see the keys up to their own positions."""
    page, T, d = 16, 40, 128
    old, new = [16, 10, 5], [20, 30, 17]
    kept = cut(new, T)
    a = make_attention(8, [o + n for o, n in zip(old, kept)], kept, 4, 2, d, page, torch.bfloat16)
    have = [-(-o // page) for o in old]
    table = torch.full_like(a["table"], -1)
    for b, h in enumerate(have):
        table[b, :h] = a["table"][b, :h]
    spare = [p for b, h in enumerate(have) for p in a["table"][b, h:].tolist() if p >= 0]
    free = spare + [0] * 8
    q_start, kv_len, _, _, nxt = P.pifa_page_tables(i32(old), i32(new), page, i32(free), i32([0]), table, T)
    assert P.pifa_device_status() == P.PIFA_ERR_CAPACITY and int(nxt) == len(spare)
    O = attend(dict(a, table=table, q_start=q_start, kv_len=kv_len))
    check_attention(a, O, d ** -0.5)


@pytest.mark.parametrize("T", [0, 1, 40])
@pytest.mark.parametrize("given", [False, True])
def test_no_requests(T, given):
    empty = lambda n, dtype=torch.int32: torch.full((n,), -3, dtype=dtype, device=DEV)
    out = (empty(1), empty(0), empty(T), empty(T, torch.int64), empty(1)) if given else None
    if not given:  # memory that the call's outputs are likely to get
        before = [empty(n, dt) for n in (1, 1, T, T) for dt in (torch.int32, torch.int64)]
        del before
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    got = P.pifa_page_tables(none, none, 16, i32([4, 5, 6]), i32([2]), torch.empty((0, 3), dtype=torch.int32, device=DEV), T, out=out)
    assert [x.tolist() for x in got] == [[0], [], [0] * T, [-1] * T, [2]]
