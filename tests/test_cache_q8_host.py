"""The cache in 8 bits without a GPU: what the C ABI and the binding refuse before anything is launched."""
import pytest
import torch

from paper_2501_19090_gb300 import pifa as P

bf16, i32, i64, e4m3, e8m0 = torch.bfloat16, torch.int32, torch.int64, torch.float8_e4m3fn, torch.float8_e8m0fnu
A = [(k + 1) << 36 for k in range(14)]  # raw addresses that no call gets as far as using, 64 GiB apart


@pytest.fixture(scope="module")
def lib():
    return P.load()


def status(name):
    return getattr(P, "PIFA_OK" if name == "OK" else "PIFA_ERR_" + name)


def write(lib, **kw):
    a = dict(Q=A[0], ldq=256, K=A[1], ldk=128, V=A[2], ldv=128, T=4, hq=2, hk=1, dim=128, dtype=0, pos=A[3], slots=A[4], freq=A[5],
             rot=128, layout=0, scale=1.0, Qr=A[6], ldqr=256, kc=A[7], vc=A[8], ks=A[9], vs=A[10], pages=10, page=32, ps=4096, ts=128,
             hs=128, sps=2, sbs=1, shs=1)
    a.update(kw)
    return lib.pifa_rope_cache_q8(*a.values(), None)


CACHE = [(dict(pages=0), "INVALID_ARG"), (dict(ps=4104), "ALIGNMENT"), (dict(ts=136, ps=8192), "ALIGNMENT"), (dict(ts=-16), "INVALID_ARG"), (dict(ts=64), "INVALID_ARG"),
         (dict(ps=2048), "INVALID_ARG"), (dict(page=8, ps=1024), "UNSUPPORTED"), (dict(sps=1), "INVALID_ARG"),
         (dict(sbs=0), "INVALID_ARG"), (dict(sps=-2), "INVALID_ARG"), (dict(sbs=1 << 47), "INVALID_ARG"),
         (dict(hk=2, ts=256, ps=8192, ldk=256, ldv=256, shs=0), "INVALID_ARG"), (dict(hk=2, ts=256, ps=8192, ldk=256, ldv=256), "INVALID_ARG"),
         (dict(kc=None), "INVALID_ARG"), (dict(vs=None), "INVALID_ARG"), (dict(vc=A[8] + 8), "ALIGNMENT")]


@pytest.mark.parametrize("kw,want", CACHE + [
    (dict(page=24, sps=1), "UNSUPPORTED"), (dict(hk=0), "INVALID_ARG"), (dict(ldk=120), "INVALID_ARG"), (dict(V=A[2] + 2), "ALIGNMENT"),
    (dict(vc=A[7]), "INVALID_ARG"), (dict(vs=A[9]), "INVALID_ARG"), (dict(Qr=A[7] + 256), "INVALID_ARG"), (dict(Qr=A[0] + 16), "INVALID_ARG"),
    (dict(K=A[7]), "INVALID_ARG"), (dict(ks=A[2]), "INVALID_ARG"), (dict(Qr=A[10]), "INVALID_ARG"), (dict(Qr=A[0], K=A[0] + 128), "INVALID_ARG"),
    (dict(rot=24), "UNSUPPORTED"), (dict(dtype=2), "INVALID_ARG"), (dict(slots=None), "INVALID_ARG"), (dict(T=-1), "INVALID_ARG"),
    (dict(T=0, Q=None, kc=None), "OK")])
def test_write_refuses(lib, kw, want):
    assert write(lib, **kw) == status(want), P.pifa_last_error()


def read(lib, **kw):
    a = dict(kc=A[7], vc=A[8], ks=A[9], vs=A[10], pages=10, page=32, hk=1, dim=128, ps=4096, ts=128, hs=128, sps=2, sbs=1, shs=1,
             slots=A[4], T=4, dtype=0, K=A[1], ldk=128, V=A[2], ldv=128)
    a.update(kw)
    return lib.pifa_cache_read_q8(*a.values(), None)


@pytest.mark.parametrize("kw,want", CACHE + [
    (dict(T=-1), "INVALID_ARG"), (dict(T=1 << 30), "INVALID_ARG"), (dict(dtype=3), "INVALID_ARG"), (dict(dim=120), "UNSUPPORTED"),
    (dict(dim=528, ts=528, ps=528 * 32, ldk=528, ldv=528), "UNSUPPORTED"), (dict(K=None), "INVALID_ARG"), (dict(slots=None), "INVALID_ARG"),
    (dict(ldv=120), "INVALID_ARG"), (dict(ldk=132), "ALIGNMENT"), (dict(K=A[1] + 8), "ALIGNMENT"), (dict(V=A[1]), "INVALID_ARG"),
    (dict(V=A[1] + 128, ldk=256, ldv=256), "INVALID_ARG"), (dict(K=A[7] + 16), "INVALID_ARG"), (dict(V=A[10]), "INVALID_ARG"),
    (dict(K=A[4]), "INVALID_ARG"), (dict(T=0, K=None), "OK")])
def test_read_refuses(lib, kw, want):
    assert read(lib, **kw) == status(want), P.pifa_last_error()


def attention(lib, **kw):
    a = dict(Q=A[0], ldq=512, T=4, hq=4, hk=1, dim=128, dtype=0, kc=A[7], vc=A[8], ks=A[9], vs=A[10], pages=10, page=32, ps=4096, ts=128,
             hs=128, sps=2, sbs=1, shs=1, table=A[3], cols=8, ldt=8, q_start=A[4], kv_len=A[5], B=4, max_q=1, scale=0.1, O=A[6], ldo=512,
             ws=A[11], ws_bytes=1 << 34)
    a.update({k: v for k, v in kw.items() if k in a})
    return lib.pifa_paged_attention_q8(*a.values(), None)


@pytest.mark.parametrize("kw,want", CACHE + [
    (dict(hq=3, hk=2), "INVALID_ARG"), (dict(max_q=0), "INVALID_ARG"), (dict(dim=96), "UNSUPPORTED"), (dict(B=4097), "UNSUPPORTED"),
    (dict(dtype=5), "INVALID_ARG"), (dict(page=48, ps=6144, sps=3), "UNSUPPORTED"), (dict(page=512, ps=1 << 16, sps=32), "UNSUPPORTED"),
    (dict(ldt=7), "INVALID_ARG"), (dict(ks=None), "INVALID_ARG"), (dict(ldq=516), "ALIGNMENT"), (dict(ws=None), "WORKSPACE"),
    (dict(ws_bytes=255), "WORKSPACE"), (dict(O=A[9]), "INVALID_ARG"), (dict(ws=A[10] - (A[10] & 255)), "INVALID_ARG"),
    (dict(O=A[7] + 1024), "INVALID_ARG"), (dict(T=0), "OK"), (dict(B=0), "OK")])
def test_attention_refuses(lib, kw, want):
    assert attention(lib, **kw) == status(want), P.pifa_last_error()


def test_binding_wants_cuda_tensors_and_the_types(lib):
    z = lambda *shape, dtype=bf16: torch.empty(shape, dtype=dtype)
    kc, ks = z(4, 32, 2, 64, dtype=e4m3), z(4, 2, 2, dtype=e8m0)
    with pytest.raises(ValueError, match="Q must be a CUDA tensor"):
        P.pifa_rope_cache_q8(z(2, 4, 64), z(2, 2, 64), z(2, 2, 64), z(2, dtype=i32), z(2, dtype=i64), z(32, dtype=i64), kc, kc.clone(), ks, ks.clone())
    with pytest.raises(ValueError, match="Q must be a CUDA tensor"):
        P.pifa_paged_attention_q8(z(2, 4, 64), kc, kc.clone(), ks, ks.clone(), z(2, 4, dtype=i32), z(3, dtype=i32), z(2, dtype=i32), 1)
    with pytest.raises(ValueError, match="k_cache must be a CUDA tensor"):
        P.pifa_cache_read_q8(kc, kc.clone(), ks, ks.clone(), z(2, dtype=i64))
    for cache in (z(4, 32, 2, 64), kc.view(torch.uint8), z(4, 32, 2, 64, dtype=torch.float8_e5m2)):
        with pytest.raises(ValueError, match="k_cache must be"):
            P._cache_strides(cache, cache.clone(), 64, e4m3, torch.device("cpu"))
    assert P._scale_strides(ks, ks.clone(), kc) == (4, 2, 1)
    turned = z(2, 4, 2, dtype=e8m0).transpose(0, 1)
    assert P._scale_strides(turned, turned.clone(memory_format=torch.preserve_format), kc) == (2, 8, 1)
    for a, b in ((ks.view(torch.uint8), ks), (z(4, 2, 1, dtype=e8m0), ks), (ks, z(4, 4, 2, dtype=e8m0)), (ks, turned), (None, ks),
                 (z(4, 2, 2, dtype=torch.float32), ks)):
        with pytest.raises(ValueError, match="_scale"):
            P._scale_strides(a, b, kc)
    with pytest.raises(ValueError, match="multiple of 16"):
        P._scale_strides(ks, ks, z(4, 24, 2, 64, dtype=e4m3))
