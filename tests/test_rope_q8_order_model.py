"""A model, on the CPU, of how the lanes that write a block of the cache in 8 bits read its scale and replace it (rope_q8.cu,
store_blocks).

Every lane needs the scale that the block had: those whose scale rises round their share of the elements that are kept to the new
one, and one lane stores that. A load may take place any time before its value is used, and lanes are not in step, so that only a
barrier between the loads and the store keeps a lane from reading the new scale for the old one, and leaving its share as it was.

The model runs lanes in random order with and without the barrier; that the kernel has it, for one warp and for several, is read from
its source.
"""
import os
import random
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_19090_gb300", "csrc", "rope_q8.cu")


def shares_left(rng, lanes, was, fresh, barrier):
    """One random schedule: how many lanes left their share in units of the old scale."""
    scale = was
    programs = {l: ["load", "round", "arrive"] + (["store"] if l == 0 else []) for l in range(lanes)}
    old, left, arrived = {}, 0, 0
    while any(programs.values()):
        lane = rng.choice([l for l, p in programs.items() if p])
        step = programs[lane][0]
        if step == "store" and barrier and arrived < lanes:
            continue
        programs[lane].pop(0)
        if step == "load":
            old[lane] = scale
        elif step == "round":
            left += not max(fresh, old[lane]) > old[lane]
        elif step == "arrive":
            arrived += 1
        else:
            scale = max(fresh, old[lane])
    return left


@pytest.mark.parametrize("lanes", [32, 64, 256])
def test_with_a_barrier_every_share_is_rounded_anew(lanes):
    rng = random.Random(lanes)
    assert sum(shares_left(rng, lanes, 120, 121, True) for _ in range(50)) == 0


def test_without_it_some_are_left():
    rng = random.Random(1)
    assert sum(shares_left(rng, 32, 120, 121, False) for _ in range(200)) > 0


def test_the_kernel_has_the_barrier_for_one_warp_and_for_several():
    text = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    body = text[text.index("store_blocks("):text.index("__global__")]
    last_use = [m.end() for m in re.finditer(r"\bwas\b", body)][-1]
    store = re.search(r"\*scale\s*=", body).start()
    between = body[last_use:store]
    assert re.search(r"if (?:constexpr )?\(GW > 1\)\s*named_barrier_sync\(1 \+ group, GW \* 32\);\s*else\s+__syncwarp\(\);", between), between
