"""The default scratch of attention over a cache in 8 bits, without a GPU (allocations go to the host): a call that cannot have the
room for keys and values in 16 bits does without."""
import pytest
import torch

from paper_2501_19090_gb300 import pifa as P
from test_scratch_host import Library, Torch, attention, disjoint


@pytest.fixture
def fake(monkeypatch):
    f = Torch(monkeypatch)
    monkeypatch.setattr(P, "_no_room", {}, raising=False)
    f.limit, f.tried, f.free, host_empty = 10 ** 9, [], 0, torch.empty

    def empty(n, **kw):
        f.tried.append(n)
        if n > f.limit:
            raise torch.OutOfMemoryError("no memory")
        return host_empty(n, **kw)
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "mem_get_info", lambda dev=None: (f.free, 10 ** 12))
    return f


def q8(least, need, stream=5):
    return P._attention_q8_workspace(least, need, 0, stream, None)


def test_the_room_is_kept_for_the_stream(fake):
    small = q8(1000, 1000)
    assert small[0] % 256 == 0 and small[1] >= 1000 and attention(1000) == small[:2]
    room = q8(1000, 50000)
    assert room[0] % 256 == 0 and room[1] >= 50000 and q8(1000, 50000)[:2] == q8(1000, 1000)[:2] == room[:2]
    assert disjoint(room, q8(1000, 50000, stream=6)) and fake.alive().count(True) == 2 + 1   # (`small` has a reference here)
    assert len(fake.tried) == 3


def test_a_call_without_the_room_takes_what_it_needs(fake):
    fake.limit = 20000
    least = q8(1000, 50000)
    assert 1000 <= least[1] < 50000 and attention(1000) == least[:2]
    tried = len(fake.tried)
    assert q8(1000, 60000)[:2] == least[:2] and len(fake.tried) == tried    # not asked for again, each failure costs milliseconds,
    room = q8(1000, 15000)                                                  # unless it is less,
    assert room[1] >= 15000
    fake.limit, fake.free = 10 ** 9, 49000
    assert q8(1000, 60000)[:2] == room[:2]
    fake.free = 60000                                                       # or as much has become free
    room = q8(1000, 60000)
    assert room[1] >= 60000 and q8(1000, 60000)[1] >= 60000 and not P._no_room
    fake.limit, fake.free = 500, 0
    assert q8(1000, 80000)[1] >= 60000 and q8(1000, 60000)[1] >= 60000      # what the stream has stays
    assert q8(1000, 60000, stream=5)[1] >= 60000
    for least in (2000, 1999):
        with pytest.raises(torch.OutOfMemoryError):
            q8(least, 2000, stream=7)


@pytest.mark.parametrize("limit", [10 ** 9, 20000])
def test_a_captured_call_has_the_graphs(fake, limit):
    fake.capturing, fake.pool, fake.limit = True, False, limit
    first, second = q8(1000, 50000), q8(1000, 50000)
    assert disjoint(first, second) and (first[1] >= 50000) == (limit > 50000) and first[1] >= 1000
    del first, second
    assert fake.alive() == [True, True]


def test_the_call_passes_what_it_got(fake, monkeypatch):
    sizes, bf16, i32, e4m3, e8m0 = [], torch.bfloat16, torch.int32, torch.float8_e4m3fn, torch.float8_e8m0fnu

    class Lib(Library):
        def __getattr__(self, name):
            if name == "pifa_paged_attention_q8":
                return lambda *a: sizes.append(a[-2]) or P.PIFA_OK
            return (lambda *a: 40000) if name.endswith("q8_workspace_size") else super().__getattr__(name)
    lib = Lib()
    monkeypatch.setattr(P, "_lib", lambda: lib)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    z = lambda *shape, dtype=bf16: torch.zeros(shape, dtype=torch.uint8 if dtype.itemsize == 1 else dtype).view(dtype)
    for f in (P._attention_workspace_size, P._attention_q8_workspace_size):
        f.cache_clear()
    call = lambda: P.pifa_paged_attention_q8(z(4, 2, 64), z(3, 16, 2, 64, dtype=e4m3), z(3, 16, 2, 64, dtype=e4m3), z(3, 1, 2, dtype=e8m0),
                                             z(3, 1, 2, dtype=e8m0), z(1, 3, dtype=i32), z(2, dtype=i32), z(1, dtype=i32), 4, O=z(4, 2, 64))
    call()
    P._attention_workspaces.clear()
    fake.limit = 5000
    call()
    for f in (P._attention_workspace_size, P._attention_q8_workspace_size):
        f.cache_clear()
    assert sizes[0] >= 40000 and 1000 <= sizes[1] < 40000
