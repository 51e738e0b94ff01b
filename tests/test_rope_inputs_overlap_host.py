"""The writes into a paged cache, without a GPU: outputs over the positions, slots or frequencies that the kernel reads are refused, buffers
next to them are not (their calls get as far as the launch, which fails where there is no device)."""
import pytest
import torch

from paper_2501_19090_gb300 import pifa as P

Q, K, V, QR, KC, VC, KS, VS, POS, SLOTS, FREQ = [(k + 1) << 36 for k in range(11)]
T, QROW, KROW, PAGES, PAGE = 40, 256, 128, 10, 32
BYTES = {"pos": 4 * T, "slots": 8 * T, "freq": 8 * 64, "Qr": 2 * T * QROW, "ks": PAGES * PAGE // 16, "vs": PAGES * PAGE // 16}


@pytest.fixture(scope="module")
def lib():
    return P.load()


def write_q8(lib, **kw):
    a = dict(Q=Q, ldq=QROW, K=K, ldk=KROW, V=V, ldv=KROW, T=T, hq=2, hk=1, dim=128, dtype=0, pos=POS, slots=SLOTS, freq=FREQ, rot=128, layout=0,
             scale=1.0, Qr=QR, ldqr=QROW, kc=KC, vc=VC, ks=KS, vs=VS, pages=PAGES, page=PAGE, ps=4096, ts=128, hs=128, sps=2, sbs=1, shs=1)
    a.update(kw)
    return lib.pifa_rope_cache_q8(*a.values(), None)


def write_16(lib, **kw):
    a = dict(Q=Q, ldq=QROW, K=K, ldk=KROW, V=V, ldv=KROW, T=T, hq=2, hk=1, dim=128, dtype=0, pos=POS, slots=SLOTS, freq=FREQ, rot=128, layout=0,
             scale=1.0, Qr=QR, ldqr=QROW, kc=KC, vc=VC, pages=PAGES, page=PAGE, ps=4096, ts=128, hs=128)
    a.update(kw)
    return lib.pifa_rope_cache(*a.values(), None)


WRITES = {"q8": (write_q8, 1, ("Qr", "kc", "vc", "ks", "vs")), "16": (write_16, 2, ("Qr", "kc", "vc"))}


def cases():
    for form, (call, elem, outputs) in WRITES.items():
        for out in outputs:
            for name in ("pos", "slots", "freq"):
                yield form, out, name, BYTES.get(out, PAGES * PAGE * 128 * elem)


@pytest.mark.parametrize("form,out,name,size", list(cases()))
def test_outputs_over_what_the_kernel_reads_are_refused(lib, form, out, name, size):
    call, base = WRITES[form][0], {"Qr": QR, "kc": KC, "vc": VC, "ks": KS, "vs": VS}[out]
    for at in (base, base + size - 8, base - BYTES[name] + 8):       # at its start, its last bytes, its first ones
        assert call(lib, **{name: at}) == P.PIFA_ERR_INVALID_ARG and "overlaps" in P.pifa_last_error(), (hex(at), P.pifa_last_error())


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: the call must not be launched")
@pytest.mark.parametrize("form,out,name,size", list(cases()))
def test_neighbours_are_taken(lib, form, out, name, size):
    call, base = WRITES[form][0], {"Qr": QR, "kc": KC, "vc": VC, "ks": KS, "vs": VS}[out]
    for at in (base + -(-size // 8) * 8, base - BYTES[name]):
        assert call(lib, **{name: at}) == P.PIFA_ERR_CUDA, P.pifa_last_error()
