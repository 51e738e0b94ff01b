"""csrc/steps.h, where a worker's segment of a head ends, on the host: the same header, compiled with a check of signed overflow,
over steps of attention up to the limit of 2^31 that a call accepts, against Python's whole numbers."""
import os
import random
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_19090_gb300", "csrc")
PROGRAM = r"""
#include <cstdio>
#include "steps.h"
int main() {
  int steps, s0, at, stop;
  while (std::scanf("%d %d %d %d", &steps, &s0, &at, &stop) == 4) std::printf("%d\n", pifa::segment_end(steps, s0, at, stop));
}
"""


def test_segments_end_right_up_to_2_31_steps(tmp_path):
    src, exe = tmp_path / "steps.cpp", tmp_path / "steps"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover=all", "-I", CSRC, str(src),
                    "-o", str(exe)], check=True)
    rng, cases = random.Random(1), []
    most = 2 ** 31 - 1
    for total in [1, 40, 10 ** 6, 2 ** 30, most - 1, most]:
        for _ in range(300):
            steps = min(total, rng.choice([1, 7, 2 ** 20, 2 ** 26, rng.randint(1, 2 ** 26)]))  # of a head
            first = rng.randint(0, (total - steps) // steps) * steps
            if rng.random() < 0.3:
                first = total - steps                                                         # the last head
            s0 = rng.choice([0, steps - 1, rng.randrange(steps)])
            at = first + s0
            stop = min(total, at + rng.choice([1, steps - s0, rng.randint(1, 2 ** 24), rng.randint(1, 2 ** 31)]))
            cases.append((steps, s0, at, stop))
    assert any(s0 + stop > most for _, s0, _, stop in cases)
    out = subprocess.run([str(exe)], input="\n".join("%d %d %d %d" % c for c in cases), check=True, capture_output=True, text=True).stdout
    assert [int(x) for x in out.split()] == [min(steps, s0 + stop - at) for steps, s0, at, stop in cases]


def test_both_kernels_use_it():
    for name in ("attention.cu", "attention_q8.cu"):
        text = open(os.path.join(CSRC, name)).read()
        assert re.search(r"int s1 = segment_end\(steps, s0, at, stop\);", text) and "s0 + stop" not in text, name
