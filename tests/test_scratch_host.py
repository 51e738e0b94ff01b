"""Who owns the binding's default scratch, without a GPU: torch's allocations go to the host, and its answers
about captures and pools are the test's."""
import contextlib
import ctypes
import gc
import threading
import time
import weakref

import pytest
import torch

from paper_2501_19090_gb300 import pifa as P


class Torch:
    """torch.empty on the host, keeping a weak reference to every buffer, and whether a capture runs."""

    def __init__(self, monkeypatch):
        self.capturing, self.pool, self.made, self.current, self.made_on = False, True, [], 0, []
        empty = torch.empty

        def host_empty(*shape, dtype, device):
            buf = empty(*shape, dtype=dtype)
            self.made.append(weakref.ref(buf))
            self.made_on.append(self.current)
            return buf
        monkeypatch.setattr(torch, "empty", host_empty)
        monkeypatch.setattr(P, "_captured", lambda run_on: self.capturing, raising=False)
        monkeypatch.setattr(torch.cuda, "memory_snapshot", self.snapshot)
        monkeypatch.setattr(torch.cuda, "stream", self.on)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda ptr: ptr)
        monkeypatch.setattr(P, "_stream_ptr", lambda s: self.current if s is None else ctypes.c_void_p(s))
        for name in ("_attention_workspaces", "_workspaces"):
            monkeypatch.setattr(P, name, {})
        monkeypatch.setattr(P, "_graph_scratches", [], raising=False)

    @contextlib.contextmanager
    def on(self, stream):
        before, self.current = self.current, stream
        yield
        self.current = before

    def snapshot(self):
        return [{"address": 0, "total_size": 2 ** 63, "segment_pool_id": (0, 7) if self.pool else (0, 0)}]

    def alive(self):
        gc.collect()
        return [r() is not None for r in self.made]


@pytest.fixture
def fake(monkeypatch):
    return Torch(monkeypatch)


def attention(need, stream=5):
    return P._attention_workspace(need, 0, stream, None)[:2]


def disjoint(a, b):
    return a[0] + a[1] <= b[0] or b[0] + b[1] <= a[0]


def test_attention_scratch_of_eager_calls_is_kept_for_each_stream(fake):
    a = attention(1000)
    assert a[0] % 256 == 0 and a[1] >= 1000
    assert attention(900) == a and attention(1000) == a and len(fake.made) == 1
    assert disjoint(a, attention(1000, stream=6))
    b = attention(50000)
    assert b[1] >= 50000 and attention(1000) == b


@pytest.mark.parametrize("warm", [False, True])
def test_attention_scratch_of_a_capture_is_the_graphs(fake, warm):
    """Neither what eager calls use, before or after, nor what another capture uses while its own tensors live."""
    fake.pool = False                      # (kept alive, so that addresses can be told apart)
    eager = [attention(1000)] if warm else []
    fake.capturing = True
    first = attention(1000)
    fake.capturing = False
    eager += [attention(1000), attention(70000)]
    fake.capturing = True
    second = attention(1000)
    assert all(disjoint(first, x) for x in eager + [second])
    assert disjoint(second, eager[-1])     # (the smaller one before it has been given back)


def test_attention_scratch_of_a_capture_outlives_larger_calls(fake):
    """In a graph's pool the memory is the graph's and the tensor may go; without one the tensor is kept."""
    for pool in (True, False):
        fake.pool, fake.capturing = pool, True
        fake.made.clear()
        attention(1000)
        fake.capturing = False
        attention(10 ** 6 * (2 - pool))
        assert fake.alive() == [not pool, True]


# ---- the scratch of the projections, their gradients and the accumulators ---------------------------------
def test_workspace_of_eager_calls_is_kept(fake):
    a = P.workspace(1000, "cuda:0")
    assert P.workspace(1256, "cuda:0") is a and P.workspace(1000, "cuda:0", tag="x") is not a
    assert P.workspace(5000, "cuda:0") is not a


@pytest.mark.parametrize("pool", [True, False])
@pytest.mark.parametrize("tag", ["", "backward"])
def test_workspace_of_a_capture_is_the_graphs(fake, pool, tag):
    fake.pool = pool
    eager = P.workspace(1000, "cuda:0", tag=tag)
    fake.capturing = True
    first, second = P.workspace(1000, "cuda:0", tag=tag), P.workspace(900, "cuda:0", tag=tag)
    assert len({t.data_ptr() for t in (eager, first, second)}) == 3
    fake.capturing = False
    assert P.workspace(1000, "cuda:0", tag=tag) is eager
    del first, second
    assert fake.alive() == [True, not pool, not pool]


def test_workspace_of_streams_differs(fake):
    """Also where the stream is the current one, unnamed; and the memory is allocated on the stream that uses it."""
    first = P.workspace(1000, "cuda:0")
    fake.current = 9
    second = P.workspace(1000, "cuda:0")
    assert second is not first and P.workspace(1000, "cuda:0", stream=9) is second
    third = P.workspace(1000, "cuda:0", stream=11)
    assert third is not second and third is not first
    fake.current = 0
    assert P.workspace(1000, "cuda:0") is first and P.workspace(1000, "cuda:0", stream=11) is third
    assert fake.made_on == [0, 9, 11]


class Library:
    """Entry points that take a while and note how many there were and how many ran at once."""

    def __init__(self):
        self.running, self.most, self.calls = 0, 0, 0

    def __getattr__(self, name):
        if "workspace_size" in name:
            return lambda *args: 1000

        def call(*args):
            self.running += 1
            self.calls += 1
            self.most = max(self.most, self.running)
            time.sleep(0.02)
            self.running -= 1
            return P.PIFA_OK
        return call


@pytest.mark.parametrize("what", ["forward", "grouped", "backward", "accumulate", "attention"])
def test_threads_that_share_scratch_enqueue_one_after_another(fake, monkeypatch, what):
    lib, bf16, i32 = Library(), torch.bfloat16, torch.int32
    monkeypatch.setattr(P, "_lib", lambda: lib)
    monkeypatch.setattr(P, "_operands", lambda *a, **k: (4, 16, 8, 16))
    monkeypatch.setattr(torch.Tensor, "device", torch.device("cuda:0"), raising=False)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    z = lambda *shape, dtype=bf16: torch.zeros(shape, dtype=dtype)
    X, Wp, C, piv, nonp = z(4, 16), z(8, 16), z(8, 8), z(8, dtype=i32), z(8, dtype=i32)
    P._workspace_size.cache_clear()
    P._attention_workspace_size.cache_clear()
    calls = {
        "forward": lambda: P.pifa_forward(X, Wp, C, piv, nonp, Y=z(4, 16)),
        "grouped": lambda: P.pifa_forward_grouped(1, X, Wp, C, piv, nonp, Y=z(4, 16)),
        "backward": lambda: P.pifa_backward(X, Wp, C, piv, nonp, z(4, 16)),
        "accumulate": lambda: P.pifa_m_accumulate(None, X, None, 0.5, z(16, 16, dtype=torch.float32)),
        "attention": lambda: P.pifa_paged_attention(z(4, 2, 64), z(3, 16, 2, 64), z(3, 16, 2, 64), z(1, 3, dtype=i32),
                                                      z(2, dtype=i32), z(1, dtype=i32), 4, O=z(4, 2, 64)),
    }
    threads = [threading.Thread(target=calls[what]) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    P._workspace_size.cache_clear()
    P._attention_workspace_size.cache_clear()
    assert lib.most == 1 and lib.calls == 4
