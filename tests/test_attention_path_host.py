"""Page tables, rotary positions and paged attention without a GPU: what the binding and the C ABI refuse
before anything is launched, and the host's frequencies against their formula."""
import math

import pytest
import torch

from paper_2501_19090_gb300 import pifa as P

bf16, i32, i64 = torch.bfloat16, torch.int32, torch.int64


@pytest.fixture(scope="module")
def lib():
    return P.load()


def formula(rot, base, i):
    return base ** (-2.0 * i / rot) / (2.0 * math.pi)


@pytest.mark.parametrize("rot", [2, 16, 64, 128, 512])
def test_frequencies(lib, rot):
    scale = 2.0 ** 64
    # pow and the division are good to a few units of 2^-53
    near = lambda got, want: abs(got / scale - want) <= 4e-16 * want + 2.0 ** -64
    plain = P.pifa_rope_frequencies(rot, base=10000.0).tolist()
    assert all(near(f, formula(rot, 1e4, i)) for i, f in enumerate(plain)) and plain[0] == int(scale / (2 * math.pi))
    linear = P.pifa_rope_frequencies(rot, scaling=P.PIFA_ROPE_SCALE_LINEAR, factor=4.0).tolist()
    assert all(near(f, formula(rot, 1e4, i) / 4) for i, f in enumerate(linear))
    if rot >= 4:
        b = P.pifa_rope_frequencies(rot, scaling=P.PIFA_ROPE_SCALE_BASE, factor=3.0).tolist()
        assert b[0] == plain[0] and abs(b[-1] / plain[-1] * 3.0 - 1.0) < 1e-13
    bands = P.pifa_rope_frequencies(rot, base=5e5, scaling=P.PIFA_ROPE_SCALE_BANDS, factor=8.0, original=8192.0, low=1.0,
                                    high=4.0).tolist()
    for i, f in enumerate(bands):
        t = formula(rot, 5e5, i)
        n = 8192.0 * t
        k = 1.0 if n >= 4 else 0.0 if n <= 1 else (n - 1) / 3
        assert abs(f / scale - t * (k + (1 - k) / 8)) <= 1e-14 * t + 2.0 ** -64  # frequencies are whole multiples of 2^-64
    assert all(0 < f < 2 ** 62 for f in plain + linear + bands)


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=514), dict(base=1.0), dict(base=math.nan),
                                dict(base=math.inf), dict(scaling=9), dict(scaling=P.PIFA_ROPE_SCALE_LINEAR, factor=0.5),
                                dict(scaling=P.PIFA_ROPE_SCALE_BASE, rot_dim=2, factor=2.0),
                                dict(scaling=P.PIFA_ROPE_SCALE_BANDS, factor=2.0),
                                dict(scaling=P.PIFA_ROPE_SCALE_BANDS, factor=2.0, original=100.0, low=4.0, high=4.0)])
def test_frequencies_refuse(lib, kw):
    with pytest.raises(P.PifaError, match="INVALID_ARG"):
        P.pifa_rope_frequencies(**{"rot_dim": 64, **kw})


# ---- the C ABI: raw addresses that no call gets as far as using -------------------------------------------
A = [(k + 1) << 36 for k in range(12)]  # 64 GiB apart


def tables(lib, **kw):
    a = dict(cached=A[0], new=A[1], B=4, page=16, free=A[2], n_free=100, first=A[3], table=A[4], cols=8, ldt=8, q_start=A[5],
             kv_len=A[6], positions=A[7], slots=A[8], T=32, nxt=A[9])
    a.update(kw)
    return lib.pifa_page_tables(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), "INVALID_ARG"), (dict(T=-1), "INVALID_ARG"), (dict(B=4097), "UNSUPPORTED"), (dict(page=0), "INVALID_ARG"),
    (dict(page=65537), "INVALID_ARG"), (dict(ldt=7), "INVALID_ARG"), (dict(cols=-1), "INVALID_ARG"), (dict(n_free=-1), "INVALID_ARG"),
    (dict(cached=None), "INVALID_ARG"), (dict(free=None), "INVALID_ARG"), (dict(table=None), "INVALID_ARG"),
    (dict(slots=None), "INVALID_ARG"), (dict(nxt=None), "INVALID_ARG"),
    (dict(q_start=A[4] + 64), "INVALID_ARG"), (dict(kv_len=A[0] + 4), "INVALID_ARG"), (dict(kv_len=A[1]), "INVALID_ARG"),
    (dict(slots=A[7]), "INVALID_ARG"), (dict(nxt=A[2]), "INVALID_ARG"), (dict(B=0), "OK")])
def test_page_tables_refuse(lib, kw, status):
    assert tables(lib, **kw) == getattr(P, "PIFA_OK" if status == "OK" else "PIFA_ERR_" + status), P.pifa_last_error()


def rope(lib, **kw):
    a = dict(X=A[0], T=4, heads=2, ldx=256, dim=128, dtype=P.PIFA_DTYPE_BF16, pos=A[1], freq=A[2], rot=128,
             layout=P.PIFA_ROPE_HALF, scale=1.0, inverse=0, Y=A[3], ldy=256)
    a.update(kw)
    return lib.pifa_rope(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), "INVALID_ARG"), (dict(heads=0), "INVALID_ARG"), (dict(dtype=2), "INVALID_ARG"), (dict(layout=2), "INVALID_ARG"),
    (dict(scale=math.nan), "INVALID_ARG"), (dict(rot=0), "INVALID_ARG"), (dict(rot=144), "INVALID_ARG"), (dict(rot=24), "UNSUPPORTED"),
    (dict(dim=120, rot=16), "UNSUPPORTED"), (dict(dim=528, ldx=1056, ldy=1056), "UNSUPPORTED"), (dict(X=None), "INVALID_ARG"),
    (dict(freq=None), "INVALID_ARG"), (dict(ldx=248), "INVALID_ARG"), (dict(ldy=260), "ALIGNMENT"), (dict(X=A[0] + 8), "ALIGNMENT"),
    (dict(Y=A[0] + 16), "INVALID_ARG"), (dict(Y=A[0], ldy=264), "INVALID_ARG"), (dict(T=0, X=None), "OK")])
def test_rope_refuses(lib, kw, status):
    assert rope(lib, **kw) == getattr(P, "PIFA_OK" if status == "OK" else "PIFA_ERR_" + status), P.pifa_last_error()


def rope_cache(lib, **kw):
    a = dict(Q=A[0], ldq=256, K=A[1], ldk=128, V=A[2], ldv=128, T=4, hq=2, hk=1, dim=128, dtype=0, pos=A[3], slots=A[4], freq=A[5],
             rot=128, layout=0, scale=1.0, Qr=A[6], ldqr=256, kc=A[7], vc=A[8], pages=10, page=16, ps=2048, ts=128, hs=128)
    a.update(kw)
    return lib.pifa_rope_cache(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(hk=0), "INVALID_ARG"), (dict(pages=0), "INVALID_ARG"), (dict(ps=2044), "ALIGNMENT"), (dict(ts=-8), "INVALID_ARG"),
    (dict(ts=64), "INVALID_ARG"), (dict(ps=1024), "INVALID_ARG"), (dict(hk=2, ldk=256, ldv=256), "INVALID_ARG"),
    (dict(ldk=120), "INVALID_ARG"), (dict(V=A[2] + 2), "ALIGNMENT"), (dict(vc=None), "INVALID_ARG"), (dict(vc=A[7]), "INVALID_ARG"),
    (dict(Qr=A[7] + 256), "INVALID_ARG"), (dict(Qr=A[0] + 16), "INVALID_ARG"), (dict(K=A[7]), "INVALID_ARG"), (dict(page=0), "INVALID_ARG"),
    (dict(T=0, Q=None), "OK")])
def test_rope_cache_refuses(lib, kw, status):
    assert rope_cache(lib, **kw) == getattr(P, "PIFA_OK" if status == "OK" else "PIFA_ERR_" + status), P.pifa_last_error()


def attention(lib, **kw):
    a = dict(Q=A[0], ldq=512, T=4, hq=4, hk=2, dim=128, dtype=0, kc=A[1], vc=A[2], pages=10, page=16, ps=4096, ts=256, hs=128,
             table=A[3], cols=8, ldt=8, q_start=A[4], kv_len=A[5], B=4, max_q=1, scale=0.1, O=A[6], ldo=512, ws=A[7], ws_bytes=1 << 34)
    a.update(kw)
    return lib.pifa_paged_attention(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), "INVALID_ARG"), (dict(hq=3), "INVALID_ARG"), (dict(hk=0), "INVALID_ARG"), (dict(max_q=0), "INVALID_ARG"),
    (dict(hq=130, hk=2, ldq=16640, ldo=16640), "UNSUPPORTED"), (dict(dim=96), "UNSUPPORTED"), (dict(B=4097), "UNSUPPORTED"),
    (dict(dtype=5), "INVALID_ARG"), (dict(page=8, ps=2048), "UNSUPPORTED"), (dict(page=48, ps=12288), "UNSUPPORTED"),
    (dict(page=512, ps=1 << 17), "UNSUPPORTED"), (dict(ldt=7), "INVALID_ARG"), (dict(cols=1 << 28, ldt=1 << 28), "INVALID_ARG"),
    (dict(scale=math.inf), "INVALID_ARG"), (dict(Q=None), "INVALID_ARG"), (dict(table=None), "INVALID_ARG"), (dict(ldo=504), "INVALID_ARG"),
    (dict(ldq=516), "ALIGNMENT"), (dict(O=A[6] + 8), "ALIGNMENT"), (dict(ws=None), "WORKSPACE"), (dict(ws_bytes=255), "WORKSPACE"),
    (dict(ws=A[7] + 16), "ALIGNMENT"), (dict(O=A[1] + 4096), "INVALID_ARG"), (dict(ws=A[0]), "INVALID_ARG"), (dict(O=A[0]), "INVALID_ARG"),
    (dict(T=0), "OK"), (dict(B=0), "OK")])
def test_attention_refuses(lib, kw, status):
    assert attention(lib, **kw) == getattr(P, "PIFA_OK" if status == "OK" else "PIFA_ERR_" + status), P.pifa_last_error()


# ---- the binding: host tensors, every check before the last (the device) ----------------------------------
def z(*shape, dtype=bf16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_wants_cuda_tensors():
    with pytest.raises(ValueError, match="X must be a CUDA tensor"):
        P.pifa_rope(z(2, 3, 64), z(2, dtype=i32), z(32, dtype=i64))
    with pytest.raises(ValueError, match="Q must be a CUDA tensor"):
        P.pifa_rope_cache(z(2, 3, 64), z(2, 1, 64), z(2, 1, 64), z(2, dtype=i32), z(2, dtype=i64), z(32, dtype=i64), z(4, 16, 1, 64), z(4, 16, 1, 64))
    with pytest.raises(ValueError, match="Q must be a CUDA tensor"):
        P.pifa_paged_attention(z(2, 3, 64), z(4, 16, 1, 64), z(4, 16, 1, 64), z(2, 4, dtype=i32), z(3, dtype=i32), z(2, dtype=i32), 1)
    with pytest.raises(ValueError, match="cached_len must be a CUDA tensor"):
        P.pifa_page_tables(z(2, dtype=i32), z(2, dtype=i32), 16, z(4, dtype=i32), z(1, dtype=i32), z(2, 4, dtype=i32), 4)


@pytest.mark.parametrize("X", [z(2, 3), z(2, 3, 64, dtype=torch.float32), z(2, 64, 3).transpose(1, 2), z(2, 6, 64)[:, ::2], [1]])
def test_binding_wants_rows_of_heads(X):
    with pytest.raises(ValueError, match="X"):
        P.pifa_rope(X, z(2, dtype=i32), z(32, dtype=i64))


def test_binding_checks_vectors_and_caches():
    cpu = torch.device("cpu")
    for bad in (z(3, dtype=i64), z(4, dtype=i32), z(6, dtype=i32)[::2], z(3, 1, dtype=i32), None):
        with pytest.raises(ValueError, match="positions must be"):
            P._vector("positions", bad, 3, i32, cpu)
    good = z(4, 16, 2, 64)
    assert P._cache_strides(good, good.clone(), 64, bf16, cpu) == (4, 16, 2, 2048, 128, 64)
    heads_first = z(4, 2, 16, 64).transpose(1, 2)
    assert P._cache_strides(heads_first, heads_first.clone(), 64, bf16, cpu) == (4, 16, 2, 2048, 64, 1024)
    for k, v in ((good, z(5, 16, 2, 64)), (good, heads_first), (z(4, 16, 2, 128), z(4, 16, 2, 128)), (good.half(), good.half()),
                 (z(4, 16, 2, 128)[..., ::2], z(4, 16, 2, 128)[..., ::2]), (good, None)):
        with pytest.raises(ValueError, match="_cache"):
            P._cache_strides(k, v, 64, bf16, cpu)
    for t in (z(3, 4, dtype=i32), z(2, 4, dtype=i64), z(2, 8, dtype=i32)[:, ::2], z(2, dtype=i32)):
        with pytest.raises(ValueError, match="table must be"):
            P._table_ld(t, 2, cpu)
    assert P._table_ld(z(2, 8, dtype=i32)[:, :5], 2, cpu) == 8 and P._table_ld(z(1, 5, dtype=i32), 1, cpu) == 5


def test_workspace_size_refuses(lib):
    assert P.pifa_paged_attention_workspace_size(0, 4, 2, 128, 3, 1) == 0
    assert P.pifa_paged_attention_workspace_size(8, 4, 2, 128, 3, 1) > 0
    for bad in ((8, 4, 3, 128, 3, 1), (8, 4, 2, 80, 3, 1), (8, 4, 2, 128, 5000, 1), (8, 4, 2, 128, 3, 0), (-1, 4, 2, 128, 3, 1)):
        with pytest.raises(P.PifaError):
            P.pifa_paged_attention_workspace_size(*bad)
