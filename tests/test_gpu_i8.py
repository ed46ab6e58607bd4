"""Matrices in 8 bits and their products against the formulas of include/lc_serve.h in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # half a step, of the value
LEAST = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}   # and of the smallest numbers


@pytest.fixture(scope="module")
def lc():
    from paper_2009_13003_amd import lc
    return lc


def coded(w):
    """Codes and scales of the rows of w by the formula, each 32-bit rounding made from a result in 64 bits, which products and quotients of two
    32-bit numbers round to without a second rounding that shows."""
    x = w.double()
    one = torch.ones((), dtype=torch.float64, device=w.device)
    top = x.abs().amax(1) if x.shape[1] else torch.zeros(x.shape[0], dtype=torch.float64, device=w.device)
    scale = (top * (one / 127).float().double()).float()
    scale = torch.where(scale < 2.0 ** -126, torch.zeros_like(scale), scale)
    inv = torch.where(scale > 0, (one / scale.double()).float(), torch.zeros_like(scale))
    q = torch.round((x * inv.double()[:, None]).float()).clamp(-127, 127)
    bad = ~torch.isfinite(top)
    scale[bad] = float("nan")
    q[bad] = 0
    return q.to(torch.int8), scale


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,k", [(1, 1), (3, 7), (5, 16), (2, 17), (9, 2043), (4, 2048), (3, 4097), (2, 8200), (1, 16500), (2, 40001), (2050, 33), (2100, 513), (2049, 2048), (7, 0)])
def test_quantising(lc, n, k, dtype):
    g = torch.Generator(DEV).manual_seed(n * 1000 + k)
    w = torch.randn(n, k + 3, device=DEV, generator=g).to(dtype)[:, :k]      # (rows that do not follow each other)
    got = lc.lc_i8_quantize(w)
    q, s = coded(w)
    assert got.codes.shape == (n, (k + 15) // 16 * 16)
    assert torch.equal(got.codes[:, :k], q) and torch.equal(got.scales, s)
    assert not got.codes[:, k:].any()
    for to in TYPES:
        back = lc.lc_i8_dequantize(got, to)
        assert torch.equal(back, (q.float() * s[:, None]).to(to))


def test_quantising_what_is_not_ordinary(lc):
    w = torch.randn(8, 100, device=DEV)
    w[0, 5], w[1, 99], w[2, 0] = float("inf"), float("nan"), -float("inf")
    w[3] = 0
    w[4] = 1e-40
    w[5, 1:] = 0
    w[6] *= 3e38 / w[6].abs().max()
    got = lc.lc_i8_quantize(w)
    q, s = coded(w)
    assert torch.equal(got.codes[:, :100], q) and torch.equal(got.scales.isnan(), s.isnan()) and torch.equal(got.scales.nan_to_num(-1), s.nan_to_num(-1))
    assert s[:3].isnan().all() and s[3] == s[4] == 0
    back = lc.lc_i8_dequantize(got)
    assert back[:3].isnan().all() and not back[3:5].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_into_given_buffers(lc, dtype):
    """Rows with a pitch, and nothing behind them touched."""
    w = torch.randn(5, 37, device=DEV).to(dtype)
    codes, scales = torch.full((5, 80), 77, dtype=torch.int8, device=DEV), torch.full((6,), 3.0, device=DEV)
    got = lc.lc_i8_quantize(w, out=lc.I8(codes, scales[:5], 37))
    q, s = coded(w)
    assert torch.equal(codes[:, :37], q) and not codes[:, 37:48].any() and (codes[:, 48:] == 77).all() and scales[5] == 3
    out = torch.full((5, 50), 9.0, dtype=dtype, device=DEV)
    lc.lc_i8_dequantize(got, out=out[:, :37])
    assert torch.equal(out[:, :37], (q.float() * s[:, None]).to(dtype)) and (out[:, 37:] == 9).all()


def product(q, s, r, t, bias):
    """The product of codes in 64 bits, and how far what is computed in 32 may be from it: the sum of codes is rounded once, multiplied twice, and the bias
    added, four roundings of half a step of numbers no larger than |sum| sx sw + |bias| (1.01: of their product with each other)."""
    y = torch.zeros(q.shape[0], r.shape[0], dtype=torch.float64, device=q.device)
    for at in range(0, q.shape[1], 4096):
        y += q[:, at:at + 4096].double() @ r[:, at:at + 4096].double().t().contiguous()
    y = y * s.double()[:, None] * t.double()[None]
    room = 4 * 1.01 * 2.0 ** -24 * y.abs()
    if bias is not None:
        room = room + 1.01 * 2.0 ** -24 * (y.abs() + bias.double().abs())
        y = y + bias.double()
    return y, room


SIZES = [(1, 1, 1), (1, 17, 16), (3, 16, 129), (16, 33, 512), (7, 1000, 2043), (17, 40, 300), (33, 100, 4099), (64, 65, 1000), (65, 1, 64), (100, 129, 127), (128, 128, 128),
         (129, 257, 1024), (300, 513, 2051), (1, 3000, 11008), (13, 130, 40000), (5, 3, 0), (1030, 300, 200), (260, 1100, 513),
         # each way of dealing tiles, with what is left over at every edge; one row too wide for its codes to be kept
         (300, 3001, 200), (641, 2501, 333), (1031, 2003, 130), (1901, 4099, 300), (25, 8200, 270), (1, 40, 33000), (2, 100, 6000), (70, 100, 4112)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", SIZES)
def test_products(lc, m, n, k, dtype):
    g = torch.Generator(DEV).manual_seed(m + n + k)
    x, w = torch.randn(m, k, device=DEV, generator=g).to(dtype), lc.lc_i8_quantize(0.05 * torch.randn(n, k, device=DEV, generator=g))
    bias = torch.randn(n, device=DEV, generator=g).to(dtype) if m % 2 else None
    q, s = coded(x)
    want, room = product(q, s, w.codes[:, :k], w.scales, bias)
    room = room + (1.01 * HALF[dtype] * want.abs() + LEAST[dtype] if dtype != torch.float32 else 0)
    got = lc.lc_i8_linear(x, w, bias)
    assert got.dtype == dtype and ((got.double() - want).abs() <= room).all()
    assert torch.equal(got, lc.lc_i8_matmul(lc.lc_i8_quantize(x), w, bias, dtype))


# few rows that one launch works out the codes of: one and two eights a lane, rows that share a wavefront, the last sizes that fit and the first that do not
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(2, 33, 1), (16, 1, 17), (9, 15, 100), (2, 200, 2048), (4, 31, 1030), (16, 100, 256), (2, 300, 4096), (2, 40, 4081), (2, 40, 4097), (4, 17, 2043),
                                   (8, 1024, 1024), (15, 50, 544), (15, 50, 545), (16, 2000, 511), (3, 2500, 2720), (3, 16, 2721), (17, 30, 300)])
def test_short_rows(lc, m, n, k, dtype):
    g = torch.Generator(DEV).manual_seed(m + n + k)
    x, w = torch.randn(m, k + 5, device=DEV, generator=g).to(dtype)[:, :k], lc.lc_i8_quantize(0.05 * torch.randn(n, k, device=DEV, generator=g))
    x[m // 2] = 0
    bias = torch.randn(n, device=DEV, generator=g).to(dtype)
    out = torch.full((m + 1, n + 3), 9.0, dtype=dtype, device=DEV)
    lc.lc_i8_linear(x, w, bias, out=out[:m, :n])
    assert torch.equal(out[:m, :n], lc.lc_i8_matmul(lc.lc_i8_quantize(x), w, bias, dtype)) and (out[m] == 9).all() and (out[:, n:] == 9).all()
    want, room = product(*coded(x), w.codes[:, :k], w.scales, bias)
    room = room + (1.01 * HALF[dtype] * want.abs() + LEAST[dtype] if dtype != torch.float32 else 0)
    assert ((out[:m, :n].double() - want).abs() <= room).all()
    for i in range(m):
        assert torch.equal(lc.lc_i8_linear(x[i:i + 1], w, bias)[0], out[i, :n])


@pytest.mark.parametrize("m", [1, 20, 200])
def test_extreme_codes(lc, m):
    """The largest sums there are, at the largest width; bytes behind a row of w that are not zeros; a code of -128."""
    k = 131072
    x = lc.I8(torch.full((m, k), 127, dtype=torch.int8, device=DEV), torch.ones(m, device=DEV), k)
    w = lc.I8(torch.full((3, k), 127, dtype=torch.int8, device=DEV), torch.ones(3, device=DEV), k)
    w.codes[1], w.codes[2] = -127, -128
    got = lc.lc_i8_matmul(x, w)
    want = torch.tensor([127 * 127 * k, -127 * 127 * k, -127 * 128 * k], dtype=torch.float64, device=DEV).float()
    assert torch.equal(got, want.expand(m, 3))
    k = 35
    w = lc.I8(torch.full((40, 48), 100, dtype=torch.int8, device=DEV), torch.ones(40, device=DEV), k)
    codes = torch.zeros(m, 48, dtype=torch.int8, device=DEV)
    codes[:, :k] = 3
    assert (lc.lc_i8_matmul(lc.I8(codes, torch.ones(m, device=DEV), k), w) == 300 * k).all()


@pytest.mark.parametrize("m", [2, 40, 130])
def test_rows_that_are_not_finite(lc, m):
    x = torch.randn(m, 64, device=DEV)
    x[1, 3] = float("nan")
    w = lc.lc_i8_quantize(torch.randn(20, 64, device=DEV))
    w.scales[5] = float("nan")
    y = lc.lc_i8_linear(x, w)
    assert y[1].isnan().all() and y[:, 5].isnan().all()
    rest = torch.ones_like(y, dtype=torch.bool)
    rest[1], rest[:, 5] = False, False
    assert y[rest].isfinite().all()


@pytest.mark.parametrize("m", [3, 50, 140])
def test_pitches_and_what_lies_behind(lc, m):
    n, k = 100, 90
    g = torch.Generator(DEV).manual_seed(m)
    x, bias = torch.randn(m, 2 * k, device=DEV, generator=g)[:, 1:k + 1], torch.randn(n, device=DEV, generator=g)
    codes = torch.full((n, 128), 55, dtype=torch.int8, device=DEV)
    w = lc.lc_i8_quantize(torch.randn(n, k, device=DEV, generator=g), out=lc.I8(codes, torch.empty(n, device=DEV), k))
    out = torch.full((m + 1, n + 9), 4.0, device=DEV)
    lc.lc_i8_linear(x, w, bias, out=out[:m, :n])
    assert torch.equal(out[:m, :n], lc.lc_i8_linear(x.contiguous(), w, bias)) and (out[m:] == 4).all() and (out[:, n:] == 4).all()


def test_no_rows(lc):
    w = lc.lc_i8_quantize(torch.randn(20, 64, device=DEV))
    assert lc.lc_i8_linear(torch.empty(0, 64, device=DEV), w).shape == (0, 20)
    none = lc.lc_i8_quantize(torch.empty(0, 64, device=DEV))
    assert none.n == 0 and lc.lc_i8_linear(torch.randn(4, 64, device=DEV), none).shape == (4, 0)


def test_on_another_stream_and_in_a_graph(lc):
    """On another stream than the current one; captured and replayed with other inputs, between eager calls."""
    g = torch.Generator(DEV).manual_seed(8)
    w = lc.lc_i8_quantize(torch.randn(300, 500, device=DEV, generator=g))
    for m in (2, 40, 200):
        x = torch.randn(m, 500, device=DEV, generator=g)
        want = lc.lc_i8_linear(x, w)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        got = lc.lc_i8_linear(x, w, stream=s)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(got, want)
        ws, out = lc.new_i8_workspace(m, 500), torch.empty(m, 300, device=DEV)
        with torch.cuda.stream(s):
            lc.lc_i8_linear(x, w, out=out, ws=ws)
        torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lc.lc_i8_linear(x, w, out=out, ws=ws)
        for i in range(3):
            x.copy_(torch.randn(m, 500, device=DEV, generator=g))
            graph.replay()
            got = out.clone()
            ws.fill_(255 - i)
            assert torch.equal(got, lc.lc_i8_linear(x, w))


def test_refused(lc):
    x = torch.randn(4, 64, device=DEV, requires_grad=True)
    w = lc.lc_i8_quantize(torch.randn(20, 64, device=DEV))
    with pytest.raises(AssertionError):
        lc.lc_i8_linear(x, w)
    with torch.no_grad():
        lc.lc_i8_linear(x, w)
    with pytest.raises(AssertionError):
        lc.lc_i8_linear(torch.randn(4, 63, device=DEV), w)
    with pytest.raises(lc.LcError):
        lc.lc_i8_linear(x.detach(), w, ws=torch.empty(0, dtype=torch.uint8, device=DEV))
    with pytest.raises(lc.LcError):
        lc.lc_i8_matmul(w, w, dtype=torch.float64)


@pytest.mark.parametrize("m", [1, 3, 100])
def test_a_matrix_beyond_4_gib(lc, m):
    """The last of w's rows, and of y's columns, whose codes lie beyond 2^32 bytes."""
    n, k = 70000, 65536
    w = lc.I8(torch.empty(n, k, dtype=torch.int8, device=DEV), torch.ones(n, device=DEV), k)
    g = torch.Generator(DEV).manual_seed(m)
    for at in (0, n - 200):
        w.codes[at:at + 200] = torch.randint(-127, 128, (200, k), device=DEV, generator=g).to(torch.int8)
    w.codes[200:n - 200] = 1
    x = lc.lc_i8_quantize(torch.randn(m, k, device=DEV, generator=g))
    y = lc.lc_i8_matmul(x, w)
    for at in (0, n - 200):
        want, room = product(x.codes, x.scales, w.codes[at:at + 200], w.scales[at:at + 200], None)
        assert ((y[:, at:at + 200].double() - want).abs() <= room).all()
    back = lc.lc_i8_dequantize(w, torch.bfloat16)
    assert torch.equal(back[n - 1], w.codes[n - 1].to(torch.bfloat16))
    again = lc.lc_i8_quantize(back[n - 3:])
    assert torch.equal(again.codes, coded(back[n - 3:])[0])
