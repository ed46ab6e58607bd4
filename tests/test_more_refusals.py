"""What the calls on 8-bit matrices, pages, prompts and drafted tokens refuse before anything is enqueued, and the sizes they state: host logic, no GPU needed.
Every pointer here is a number that nothing may read."""
import ctypes

import pytest

OK, BADARG, WORKSPACE = 0, 1, 6
F32, BF16, F16, F64 = range(4)
P = 1 << 20                                                 # an address that suits every alignment


@pytest.fixture(scope="module")
def lib():
    from paper_2009_13003_amd import lc
    return lc._lib


def described(struct, defaults, kw):
    a = dict(defaults, **kw)
    return ctypes.byref(struct(*(a[f] for f, _ in struct._fields_)))


def i8(**kw):
    from paper_2009_13003_amd import lc
    return described(lc._I8, dict(codes=P, scales=P, n=8, k=100, pitch=112), kw)


def kv(**kw):
    from paper_2009_13003_amd import lc
    return described(lc._KvCache, dict(k=P, v=P, k_scale=P, v_scale=P, pages=10, page_tokens=16, heads=2, dim=64, bits=8), kw)


def pages(**kw):
    from paper_2009_13003_amd import lc
    return described(lc._KvPages, dict(table=P, lens=P, free_pages=P, free_count=P, batch=2, ld_table=4, table_pages=4, free_room=10, page_tokens=16), kw)


@pytest.mark.parametrize("bad", [dict(codes=None), dict(scales=None), dict(codes=P + 8), dict(scales=P + 2), dict(pitch=96), dict(pitch=120), dict(n=1 << 31),
                                 dict(k=131073, pitch=1 << 18), dict(pitch=1 << 41)])
def test_matrices_described_wrongly(lib, bad):
    assert lib.lc_i8_quantize(P, 1 << 18, F32, i8(**bad), None) == BADARG
    assert lib.lc_i8_dequantize(i8(**bad), P, 1 << 18, F32, None) == BADARG
    assert lib.lc_i8_matmul(i8(**bad), i8(), None, P, 8, F32, None) == BADARG
    assert lib.lc_i8_matmul(i8(), i8(**bad), None, P, 8, F32, None) == BADARG
    assert lib.lc_i8_linear(P, 1 << 18, 1, i8(**bad), None, P, 8, F32, P, 1 << 30, None) == BADARG


def test_matrix_arguments(lib):
    for dtype in (F64, -1, 4):
        assert lib.lc_i8_quantize(P, 100, dtype, i8(), None) == BADARG
        assert lib.lc_i8_dequantize(i8(), P, 100, dtype, None) == BADARG
        assert lib.lc_i8_matmul(i8(), i8(), None, P, 8, dtype, None) == BADARG
        assert lib.lc_i8_linear(P, 100, 1, i8(), None, P, 8, dtype, P, 1 << 20, None) == BADARG
    for w, ld in ((None, 100), (P + 2, 100), (P, 99), (P, 1 << 41)):
        assert lib.lc_i8_quantize(w, ld, F32, i8(), None) == BADARG
        assert lib.lc_i8_dequantize(i8(), w, ld, F32, None) == BADARG
    assert lib.lc_i8_quantize(P, 100, F32, None, None) == BADARG
    ok = [i8(n=2), i8(), None, P, 8]                         # x8, w8, bias, y, ldy
    for at, value in ((0, None), (0, i8(n=2, k=99)), (0, i8(n=(1 << 19) + 1)), (1, None), (2, P + 2), (3, None), (3, P + 1), (4, 7), (4, 1 << 41)):
        a = list(ok)
        a[at] = value
        assert lib.lc_i8_matmul(*a, F32, None) == BADARG, (at, value)
    ok = [P, 100, 2, i8(), None, P, 8, F32, P, 1 << 20]
    for at, value, want in ((0, None, BADARG), (0, P + 2, BADARG), (1, 99, BADARG), (1, 1 << 41, BADARG), (2, (1 << 19) + 1, BADARG), (4, P + 1, BADARG),
                            (5, None, BADARG), (6, 7, BADARG), (8, None, WORKSPACE), (8, P + 128, WORKSPACE), (9, 255, WORKSPACE)):
        a = list(ok)
        a[at] = value
        assert lib.lc_i8_linear(*a, None) == want, (at, value)


def test_nothing_to_do(lib):
    assert lib.lc_i8_quantize(None, 0, F32, i8(n=0, codes=None, scales=None), None) == OK
    assert lib.lc_i8_dequantize(i8(k=0, codes=None), None, 0, F32, None) == OK
    assert lib.lc_i8_matmul(i8(n=0, codes=None, scales=None), i8(), None, None, 0, F32, None) == OK
    assert lib.lc_i8_linear(None, 0, 0, i8(), None, None, 0, F32, None, 0, None) == OK
    assert lib.lc_kv_attend_prompt(kv(), None, 0, 0, 2, None, 1, None, 0, 0, None, 1.0, None, 0, F32, None, 0, None) == OK
    assert lib.lc_kv_attend_prompt(kv(), None, 0, 3, 2, None, 0, None, 0, 0, None, 1.0, None, 0, F32, None, 0, None) == OK
    assert lib.lc_draft_verify(None, 0, 0, 0, 1, 1, None, None, 0, 0, None, None, None, F32, None, None, None, None, 0, None) == OK


def test_workspaces(lib):
    f = lib.lc_i8_workspace_bytes
    assert f((1 << 19) + 1, 5) == f(5, 131073) == 0
    for m, k in ((0, 0), (1, 1), (3, 100), (1 << 19, 131072)):
        assert f(m, k) % 256 == 0 and f(m, k) >= m * ((k + 15) // 16 * 16) + 4 * m
    f = lib.lc_kv_prompt_workspace_bytes
    for bad in (((1 << 24) + 1, 1, 1, 1, 64), (1, 65536, 1, 1, 64), (1, 1, 3, 2, 64), (1, 1, 0, 1, 64), (1, 1, 1, 0, 64), (1, 1, 4097, 1, 64), (1, 1, 1, 1, 48), (1, 1, 1, 1, 288),
                (1, 1, 1025, 1025, 64), (1 << 20, 1, 2048, 1024, 32)):
        assert f(*bad) == 0, bad
    for tokens in (0, 1, 100, 5000):
        for batch in (0, 1, 9, 65535):
            assert f(tokens, batch, 32, 8, 128) >= 256 and f(tokens, batch, 32, 8, 128) % 256 == 0
    assert f(100000, 1, 32, 8, 128) == 256                   # rows enough: nothing is split
    f = lib.lc_draft_workspace_bytes
    assert f(65536) == 0 and f(1) >= 64 * 16 and f(65535) >= 65535 * 64 * 16 and f(7) % 256 == 0


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=P + 4), dict(k_scale=None), dict(page_tokens=24), dict(heads=0), dict(dim=48), dict(bits=2)])
def test_caches_described_wrongly(lib, bad):
    assert lib.lc_kv_attend_prompt(kv(**bad), P, 128, 3, 2, P, 1, P, 4, 4, P, 1.0, P, 128, F32, P, 1 << 30, None) == BADARG


def test_prompt_arguments(lib):
    names = ["q", "ld_q", "tokens", "heads", "starts", "batch", "table", "ld_table", "table_pages", "lens", "scale", "out", "ld_out", "dtype", "ws", "ws_bytes"]
    ok = dict(q=P, ld_q=256, tokens=3, heads=4, starts=P, batch=2, table=P, ld_table=4, table_pages=4, lens=P, scale=1.0, out=P, ld_out=256, dtype=F32, ws=P, ws_bytes=1 << 30)
    for name, value, want in (("q", None, BADARG), ("q", P + 8, BADARG), ("ld_q", 255, BADARG), ("ld_q", 258, BADARG), ("ld_q", 1 << 41, BADARG), ("tokens", (1 << 24) + 1, BADARG),
                              ("heads", 3, BADARG), ("heads", 0, BADARG), ("heads", 4098, BADARG), ("starts", None, BADARG), ("starts", P + 2, BADARG), ("batch", 65536, BADARG),
                              ("table", None, BADARG), ("table", P + 2, BADARG), ("ld_table", 3, BADARG), ("table_pages", (1 << 26) + 1, BADARG), ("lens", None, BADARG),
                              ("lens", P + 1, BADARG), ("out", None, BADARG), ("out", P + 8, BADARG), ("ld_out", 252, BADARG), ("ld_out", 257, BADARG), ("dtype", F64, BADARG),
                              ("ws", None, WORKSPACE), ("ws", P + 128, WORKSPACE), ("ws_bytes", 255, WORKSPACE)):
        a = dict(ok)
        a[name] = value
        assert lib.lc_kv_attend_prompt(kv(), *(a[n] for n in names), None) == want, (name, value)
    a = dict(ok, dtype=BF16, ld_q=260)
    assert lib.lc_kv_attend_prompt(kv(), *(a[n] for n in names), None) == BADARG


@pytest.mark.parametrize("bad", [dict(table=None), dict(table=P + 2), dict(lens=None), dict(lens=P + 1), dict(free_pages=None), dict(free_pages=P + 2), dict(free_count=None),
                                 dict(free_count=P + 2), dict(batch=65536), dict(ld_table=3), dict(ld_table=1 << 32), dict(table_pages=(1 << 26) + 1, ld_table=1 << 27),
                                 dict(free_room=1 << 31), dict(page_tokens=24), dict(page_tokens=4), dict(page_tokens=2048), dict(page_tokens=0)])
def test_pages_described_wrongly(lib, bad):
    assert lib.lc_kv_extend(pages(**bad), P, 5, P, P, P, P, P, P, None) == BADARG
    assert lib.lc_kv_trim(pages(**bad), P, P, P, None) == BADARG


def test_page_arguments(lib):
    assert lib.lc_kv_extend(None, P, 5, P, P, P, P, P, P, None) == BADARG and lib.lc_kv_trim(None, P, P, P, None) == BADARG
    ok = [P, 5, P, P, P, P, P, P]                            # add, room, new_lens, new_count, starts, slots, places, owners
    for at, value in ((0, None), (0, P + 2), (1, 1 << 31), (2, None), (2, P + 1), (3, None), (3, P + 2), (4, None), (4, P + 2), (5, None), (5, P + 4), (6, P + 2), (7, P + 1)):
        a = list(ok)
        a[at] = value
        assert lib.lc_kv_extend(pages(), *a, None) == BADARG, (at, value)
    for a in ((None, P, P), (P + 2, P, P), (P, None, P), (P, P + 2, P), (P, P, None), (P, P, P + 2)):
        assert lib.lc_kv_trim(pages(), *a, None) == BADARG, a


def test_draft_arguments(lib):
    names = ["target", "ld_batch", "ld_row", "batch", "nodes", "vocab", "tokens", "draft", "ld_draft_batch", "ld_draft_row", "parent", "count", "uniform", "dtype", "path", "length",
             "next", "ws", "ws_bytes"]
    ok = dict(target=P, ld_batch=300, ld_row=100, batch=2, nodes=3, vocab=100, tokens=P, draft=P, ld_draft_batch=200, ld_draft_row=100, parent=None, count=P, uniform=P, dtype=F32,
              path=P, length=P, next=P, ws=P, ws_bytes=1 << 20)
    for name, value, want in (("target", None, BADARG), ("target", P + 2, BADARG), ("ld_batch", 1 << 41, BADARG), ("ld_row", 1 << 41, BADARG), ("batch", 65536, BADARG),
                              ("nodes", 0, BADARG), ("nodes", 65, BADARG), ("vocab", 0, BADARG), ("vocab", (1 << 24) + 1, BADARG), ("tokens", None, BADARG), ("tokens", P + 2, BADARG),
                              ("draft", P + 1, BADARG), ("ld_draft_batch", 1 << 41, BADARG), ("ld_draft_row", 1 << 41, BADARG), ("parent", P, BADARG), ("count", P + 2, BADARG),
                              ("uniform", None, BADARG), ("uniform", P + 2, BADARG), ("dtype", F64, BADARG), ("path", None, BADARG), ("length", P + 2, BADARG), ("next", None, BADARG),
                              ("ws", None, WORKSPACE), ("ws", P + 64, WORKSPACE), ("ws_bytes", 100, WORKSPACE)):
        a = dict(ok)
        a[name] = value
        assert lib.lc_draft_verify(*(a[n] for n in names), None) == want, (name, value)


def test_prompts_and_temperatures_of_the_decoder():
    """Refused before anything is counted or enqueued."""
    from paper_2009_13003_amd import serve
    model = serve.Decoder.__new__(serve.Decoder)
    model.batch, model.count, model.pages = 2, [0, 0], None
    with pytest.raises(ValueError, match="shared"):
        model.read_prompts([[1], [2]])
    model.pages = object()
    for prompts in ([[1]], [[1], [2], [3]], [[1], []], [[], []]):
        with pytest.raises(ValueError, match="a token or more"):
            model.read_prompts(prompts)
    for temperature in (0.0, -1.0, 1e-40, float("nan")):
        with pytest.raises(ValueError, match="temperature"):
            serve.write_on(model, [[1], [2]], 3, sample=object(), temperature=temperature)
    assert model.count == [0, 0]
