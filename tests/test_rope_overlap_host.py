"""The rotation in place, without a GPU: keys or values that are elements of Q are refused, neighbouring columns are
not (their calls get as far as the launch, which fails where there is no device)."""
import pytest
import torch

from paper_2501_19090_gb300 import pifa as P

Q, POS, SLOTS, FREQ, KC, VC = [(k + 1) << 36 for k in range(6)]
LD, QROW, KROW = 512, 256, 128   # rows of 2 query heads and 1 key, 1 value head of 128; then nothing


@pytest.fixture(scope="module")
def lib():
    return P.load()


def call(lib, K, V, ldk=LD, ldv=LD, T=4):
    return lib.pifa_rope_cache(Q, LD, K, ldk, V, ldv, T, 2, 1, 128, 0, POS, SLOTS, FREQ, 128, 0, 1.0, Q, LD, KC, VC, 10, 16, 2048, 128,
                               128, None)


FAR = 1 << 35
OVERLAP = {"keys_are_queries": (Q, FAR, {}), "values_are_queries": (FAR, Q, {}), "second_head": (Q + 2 * 128, FAR, {}),
           "columns_reach_into": (Q + 2 * 248, FAR, {}), "columns_wrap_into": (Q + 2 * 392, FAR, {}),
           "next_row": (Q + 2 * LD, FAR, {}), "rows_before": (Q - 2 * 2 * LD, FAR, {}), "another_pitch": (Q + 2 * 256, FAR, {"ldk": 640}),
           "another_pitch_before": (Q - 2 * 1280, FAR, {"ldk": 1160})}
APART = {"columns": (Q + 2 * 256, Q + 2 * 384, {}), "columns_before": (Q - 2 * 128, Q - 2 * 256, {}),
         "rows_after": (Q + 2 * 4 * LD, FAR, {}), "elsewhere": (FAR, FAR + (1 << 30), {}), "one_row": (Q + 2 * 256, Q + 2 * LD, {"T": 1}),
         "other_pitch_elsewhere": (FAR, FAR + (1 << 30), {"ldk": 128, "ldv": 136})}


@pytest.mark.parametrize("name", list(OVERLAP))
def test_shared_elements_are_refused(lib, name):
    K, V, kw = OVERLAP[name]
    assert call(lib, K, V, **kw) == P.PIFA_ERR_INVALID_ARG and "overlaps" in P.pifa_last_error()


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: the call must not be launched")
@pytest.mark.parametrize("name", list(APART))
def test_other_columns_and_rows_are_taken(lib, name):
    K, V, kw = APART[name]
    assert call(lib, K, V, **kw) == P.PIFA_ERR_CUDA
