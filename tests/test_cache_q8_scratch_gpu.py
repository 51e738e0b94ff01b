"""The default scratch of attention over a cache in 8 bits: the room for 16 bits is done without where there is no memory for it."""
import pytest
import torch

from paper_2501_19090_gb300 import pifa as P
from test_cache_q8_gpu import attend, make_q8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_a_long_chunk_without_memory_for_the_room():
    a = make_q8(3, [40000], [130], 64, 8, 128, 64, torch.bfloat16)     # 164 MB of keys and values in 16 bits
    without, with_room = attend(a, room=False), attend(a, room=True)
    assert a["wide"] and not torch.equal(without, with_room)           # (weights of another type)
    torch.cuda.synchronize()
    P._attention_workspaces.clear()
    torch.cuda.empty_cache()
    total = torch.cuda.get_device_properties(0).total_memory
    P._no_room.clear()
    try:
        torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + 120 * 2 ** 20) / total)
        for _ in range(2):
            assert torch.equal(attend(a), without) and len(P._no_room) == 1
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    P._no_room.clear()
    assert torch.equal(attend(a), with_room)
    assert P.pifa_device_status() == P.PIFA_OK
