"""A block of values whose scale is NaN: NaN for the rows that see a token of it, nothing for the others, whichever kernel a call takes."""
import pytest
import torch

from paper_2501_19090_gb300 import pifa as P
from test_attention_path_gpu import plain_attention
from test_cache_q8_gpu import DTYPES, U, U8, attend, make_q8, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,room", [(2, False), (6, False), (40, False), (400, False), (400, True), (900, True)])
def test_scale_of_nan_stays_with_the_rows_that_see_it(new, room, dtype, d):
    """Blocks of the cached tokens, of the new ones, and the last one, of keys' and of values' scales; the other heads and requests as if there
    were none, and rows that see none of it within the bounds of the formula (the tile's largest scale may be another one)."""
    L, hq, hk, page = 260 + new, 6, 2, 32
    a = make_q8(13, [L, 90], [new, 1], hq, hk, d, page, dtype)
    good = attend(a, room=room)
    assert a["wide"] == (room and new * 3 > 768)
    want, size, keys = plain_attention(a, d ** -0.5)
    w = U[dtype] if a["wide"] else 2.0 ** -11
    tol = U[dtype] * want.abs() + (1.1 * w + 2e-4) * size + 2.0 ** -24 * (1.0 + keys) * float(values(a["v8"], a["vs"])[a["table"][0, :L // page].long()].abs().max())
    for name, elements in (("vs", False), ("vs", True), ("ks", False)):
        for at in (5, 260 + new // 2, L - 1):
            b = dict(a, k8=a["k8"].clone(), v8=a["v8"].clone(), ks=a["ks"].clone(), vs=a["vs"].clone())
            block, p = at // 16 * 16, int(a["table"][0, at // page])
            b[name].view(U8)[p, at % page // 16, 1] = 0xff
            if elements:                                       # as memory that nobody has written may have it
                b["v8"].view(U8)[p, block % page:][:16, 1] = 0x7f
            O = attend(b, room=room)
            assert P.pifa_device_status() == P.PIFA_OK
            first = max(0, block - (L - new))                  # the first new token that sees a key of the block
            assert bool(O[first:new, 3:].isnan().all())
            assert torch.equal(O[:new, :3], good[:new, :3]) and torch.equal(O[new:], good[new:])
            err = (O[:first].double() - want[:first]).abs()
            assert bool((err <= tol[:first]).all()), (name, at, int((~(err <= tol[:first])).sum()))
