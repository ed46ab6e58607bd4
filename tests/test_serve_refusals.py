"""What the calls of include/lc_serve.h refuse before anything is enqueued, and the sizes they state: host logic, no GPU needed.
Every pointer here is a number that nothing may read."""
import ctypes
import os

import pytest

OK, BADARG, WORKSPACE = 0, 1, 6
F32, BF16, F16, F64 = range(4)
P = 1 << 20                                                 # an address that suits every alignment


@pytest.fixture(scope="module")
def lib():
    from paper_2009_13003_amd import lc
    return lc._lib


def w4(**kw):
    from paper_2009_13003_amd import lc
    a = dict(codes=P, scales=P, n=8, k=100, codes_pitch=64, scales_pitch=4, group=32)
    a.update(kw)
    return ctypes.byref(lc._W4(*(a[f] for f, _ in lc._W4._fields_)))


def kv(**kw):
    from paper_2009_13003_amd import lc
    a = dict(k=P, v=P, k_scale=P, v_scale=P, pages=10, page_tokens=16, heads=2, dim=64, bits=8)
    a.update(kw)
    return ctypes.byref(lc._KvCache(*(a[f] for f, _ in lc._KvCache._fields_)))


def test_row_bytes(lib):
    assert [lib.lc_w4_row_bytes(k) for k in (0, 1, 32, 33, 4096, (1 << 31) - 1, 1 << 31)] == [0, 16, 16, 32, 2048, 1 << 30, 0]


BAD_W4 = [dict(codes=None), dict(scales=None), dict(codes=P + 8), dict(scales=P + 1), dict(codes_pitch=48), dict(codes_pitch=72), dict(scales_pitch=3),
          dict(group=16), dict(group=0), dict(group=-32), dict(n=1 << 31), dict(k=1 << 31), dict(codes_pitch=1 << 41)]


@pytest.mark.parametrize("bad", BAD_W4)
def test_weights_described_wrongly(lib, bad):
    assert lib.lc_w4_quantize(P, 100, F32, w4(**bad), None) == BADARG
    assert lib.lc_w4_dequantize(w4(**bad), P, 100, F32, None) == BADARG
    assert lib.lc_w4_matmul(P, 100, 1, w4(**bad), None, P, 8, F32, None) == BADARG


def test_weights_arguments(lib):
    for dtype in (F64, -1, 4):
        assert lib.lc_w4_quantize(P, 100, dtype, w4(), None) == BADARG
        assert lib.lc_w4_dequantize(w4(), P, 100, dtype, None) == BADARG
        assert lib.lc_w4_matmul(P, 100, 1, w4(), None, P, 8, dtype, None) == BADARG
    assert lib.lc_w4_quantize(P, 100, F32, None, None) == BADARG
    assert lib.lc_w4_quantize(None, 100, F32, w4(), None) == BADARG
    assert lib.lc_w4_quantize(P, 99, F32, w4(), None) == BADARG
    assert lib.lc_w4_quantize(P + 2, 100, F32, w4(), None) == BADARG
    assert lib.lc_w4_dequantize(w4(), None, 100, F32, None) == BADARG
    assert lib.lc_w4_dequantize(w4(), P + 1, 100, BF16, None) == BADARG
    ok = [P, 100, 1, None, P, 8]                             # x, ldx, m, bias, y, ldy
    for at, value in ((0, None), (0, P + 2), (1, 99), (2, (1 << 19) + 1), (3, P + 1), (4, None), (4, P + 2), (5, 7), (1, 1 << 41), (5, 1 << 41)):
        a = list(ok)
        a[at] = value
        assert lib.lc_w4_matmul(a[0], a[1], a[2], w4(), a[3], a[4], a[5], F32, None) == BADARG, (at, value)


def test_nothing_to_do(lib):
    assert lib.lc_w4_quantize(None, 0, F32, w4(n=0, codes=None, scales=None), None) == OK
    assert lib.lc_w4_quantize(None, 0, F32, w4(k=0, codes=None, scales=None), None) == OK
    assert lib.lc_w4_matmul(None, 0, 0, w4(), None, None, 0, F32, None) == OK
    assert lib.lc_kv_write(kv(), None, None, 0, 0, None, 0, F32, None) == OK
    assert lib.lc_kv_read(kv(), None, 0, None, None, 0, 0, F32, None) == OK
    assert lib.lc_kv_attend(kv(), None, 0, 1, 2, None, 0, 0, None, None, 1.0, None, F32, None, 0, None) == OK


BAD_KV = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=P + 8), dict(v=P + 4), dict(k_scale=P + 4), dict(v_scale=P + 8),
          dict(page_tokens=4), dict(page_tokens=24), dict(page_tokens=2048), dict(page_tokens=-16), dict(pages=(1 << 27) + 1), dict(heads=0), dict(heads=1025),
          dict(dim=0), dict(dim=48), dict(dim=288), dict(bits=2), dict(bits=16)]


@pytest.mark.parametrize("bad", BAD_KV)
def test_caches_described_wrongly(lib, bad):
    assert lib.lc_kv_write(kv(**bad), P, P, 128, 64, P, 1, F32, None) == BADARG
    assert lib.lc_kv_read(kv(**bad), P, 1, P, P, 128, 64, F32, None) == BADARG
    assert lib.lc_kv_attend(kv(**bad), P, 1, 1, 2, P, 4, 4, P, None, 1.0, P, F32, P, 1 << 30, None) == BADARG


def test_cache_arguments(lib):
    ok = [P, P, 128, 64, P, 3]                               # k, v, ld_token, ld_head, slots, tokens
    for at, value in ((0, None), (1, None), (0, P + 2), (1, P + 1), (2, 63), (3, 63), (4, None), (4, P + 4), (5, (1 << 31) + 1), (2, 1 << 41), (3, 1 << 41)):
        a = list(ok)
        a[at] = value
        assert lib.lc_kv_write(kv(), *a, F32, None) == BADARG, (at, value)
        assert lib.lc_kv_read(kv(), a[4], a[5], a[0], a[1], a[2], a[3], F32, None) == BADARG, (at, value)
    for dtype in (F64, -1, 4):
        assert lib.lc_kv_write(kv(), *ok, dtype, None) == BADARG
        assert lib.lc_kv_read(kv(), P, 3, P, P, 128, 64, dtype, None) == BADARG


def test_attention_arguments(lib):
    names = ["q", "batch", "nq", "heads", "table", "ld_table", "table_pages", "lens", "mask", "scale", "out", "dtype", "ws", "ws_bytes"]
    ok = dict(q=P, batch=2, nq=3, heads=4, table=P, ld_table=4, table_pages=4, lens=P, mask=P, scale=1.0, out=P, dtype=F32, ws=P, ws_bytes=1 << 30)
    for name, value, want in (("q", None, BADARG), ("q", P + 8, BADARG), ("out", None, BADARG), ("out", P + 8, BADARG), ("lens", None, BADARG),
                              ("lens", P + 2, BADARG), ("table", None, BADARG), ("table", P + 2, BADARG), ("mask", P + 4, BADARG), ("ld_table", 3, BADARG),
                              ("table_pages", (1 << 26) + 1, BADARG), ("nq", 0, BADARG), ("nq", 65, BADARG), ("heads", 3, BADARG), ("heads", 0, BADARG),
                              ("heads", 4098, BADARG), ("batch", 65536, BADARG), ("dtype", F64, BADARG), ("ws", None, WORKSPACE), ("ws", P + 128, WORKSPACE),
                              ("ws_bytes", 255, WORKSPACE)):
        a = dict(ok)
        a[name] = value
        assert lib.lc_kv_attend(kv(), *(a[n] for n in names), None) == want, (name, value)


def test_workspace_bytes(lib):
    f = lib.lc_kv_workspace_bytes
    for bad in ((65536, 1, 1, 1, 64), (1, 0, 1, 1, 64), (1, 65, 1, 1, 64), (1, 1, 3, 2, 64), (1, 1, 0, 1, 64), (1, 1, 1, 0, 64), (1, 1, 4097, 1, 64),
                (1, 1, 1, 1, 48), (1, 1, 1, 1, 0), (1, 1, 1, 1, 288)):
        assert f(*bad) == 0, bad
    for batch in (1, 3, 17, 65535):
        for nq in (1, 24, 64):
            for heads, kvh in ((1, 1), (32, 8), (32, 32)):
                size = f(batch, nq, heads, kvh, 128)
                assert size >= 256 and size % 256 == 0
                assert size <= 256 + batch * nq * heads * 64 * (128 + 2) * 4 + 256          # never more than 64 parts a row
