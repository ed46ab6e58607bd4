"""Attention of many new tokens a sequence over the cache, against the formula of include/lc_serve.h in 64 bits over what the cache holds."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def lc():
    from paper_2009_13003_amd import lc
    return lc


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def filled(lc, seed, lens, kv, dim, bits, page, spare=3, spread=1.0):
    """A cache whose pages lie in any order, with whatever in what no sequence has."""
    g = torch.Generator(DEV).manual_seed(seed)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    cache = lc.new_kv_cache(pages, kv, page, dim, bits)
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(0, 256, t.shape, dtype=torch.uint8, device=DEV, generator=g))
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(float("nan"))
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    table, at = torch.full((len(lens), max(need + [1])), 10 ** 9, dtype=torch.int32), 0
    slots = []
    for b, n in enumerate(lens):
        table[b, :need[b]] = torch.tensor(order[at:at + need[b]], dtype=torch.int32)
        slots += [int(table[b, t // page]) * page + t % page for t in range(n)]
        at += need[b]
    k, v = (spread * torch.randn(len(slots), kv, dim, device=DEV, generator=g) for _ in range(2))
    lc.lc_kv_write(cache, k, v, torch.tensor(slots, dtype=torch.int64, device=DEV))
    return cache, table.to(DEV)


def want_of(lc, cache, q, starts, table, lens, scale=None):
    """Results in 64 bits and how far the kernel's may be from them:
      scores      q . k of dim terms added up in 32 bits in steps of 16, then scale and key's scale: (dim / 16 + 16 + 4) half steps of |q| . |k| times both at most;
                  exp2 and what scores are measured from: 4 half steps of the score and 4 more; both the numerator's and the sum's
      products    sums over n tokens in steps of 16, joined: n / 16 + 64 half steps of the sum of p |v|
      roundings   of p times the value's scale to fp16 (2^-11, and 2^-35 of the largest so far), in fp32 in three parts 2^-23
      the result  half a step of its type, and of its smallest numbers"""
    dtype, (_, heads, dim), g = q.dtype, q.shape, q.shape[1] // cache.heads
    out, room = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    scale = dim ** -0.5 if scale is None else scale
    page = cache.page_tokens
    eps = 2.0 ** -24
    for b, n in enumerate(lens):
        first, count = starts[b], starts[b + 1] - starts[b]
        if count <= 0 or n <= 0:
            continue
        slots = [int(table[b, t // page]) * page + t % page if 0 <= int(table[b, t // page]) < cache.pages else -1 for t in range(n)]
        there = torch.tensor([s >= 0 for s in slots], device=DEV)
        k, v = (t.double() for t in lc.lc_kv_read(cache, torch.tensor(slots, dtype=torch.int64, device=DEV)))
        # (values read back are fl32(code * scale): half a step of their own)
        last = n - count + torch.arange(count, device=DEV)
        seen = (torch.arange(n, device=DEV)[None] <= last[:, None]) & there[None]
        for h in range(heads):
            x, kk, vv = q[first:first + count, h].double(), k[:, h // g], v[:, h // g]
            score = ((x @ kk.T) * scale).masked_fill(~seen, -math.inf)
            p = torch.softmax(score, -1).nan_to_num(0.0) if not score.isnan().any() else torch.softmax(score, -1)
            p = torch.where(seen.any(1, keepdim=True), p, torch.zeros_like(p))
            nan = (seen[:, :, None] & vv.isnan()[None]).any(1)
            o = torch.where(nan, math.nan, p @ vv.nan_to_num(0.0))
            size = ((x.abs() @ kk.abs().T) * abs(scale)).masked_fill(~seen, 0.0)
            far = 2 * ((dim / 16 + 20) * size.amax(1) + 4 * score.abs().nan_to_num(0.0, 0.0, 0.0).amax(1) + 4) * eps
            carried = p.nan_to_num(0.0) @ vv.abs().nan_to_num(0.0)
            each = {torch.float32: 2.0 ** -23, torch.bfloat16: 2.0 ** -11, torch.float16: 2.0 ** -11}[dtype]
            r = carried * (far[:, None] + (n / 16 + 64) * eps + each) * 1.01
            if dtype != torch.float32:                       # (codes of 127 at most; a row's tiles reach 63 tokens beyond it)
                r = r + seen.sum(1, keepdim=True) * 2.0 ** -35 * 16 * vv.abs().nan_to_num(0.0).max()
            out[first:first + count, h] = o
            room[first:first + count, h] = r + HALF[dtype] * 1.01 * o.abs().nan_to_num(0.0) + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -133)
    return out, room


def check(got, want, room):
    assert torch.equal(got.isnan(), want.isnan())
    bad = ~((got.double() - want).abs() <= room) & ~want.isnan()
    assert not bad.any(), ((got.double() - want).abs() / room).nan_to_num(0.0).max().item()


def run(lc, seed, new, lens, heads, kv, dim, bits, dtype, page, scale=None):
    cache, table = filled(lc, seed, lens, kv, dim, bits, page)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    g = torch.Generator(DEV).manual_seed(seed + 1)
    q = (1.5 * torch.randn(starts[-1], heads, dim, device=DEV, generator=g)).to(dtype)
    got = lc.lc_kv_attend_prompt(cache, q, ints(starts), table, ints(lens), scale)
    check(got, *want_of(lc, cache, q, starts, table, lens, scale))


SHAPES = [([1], [1], 1, 1, 32, 8), ([1], [300], 4, 2, 64, 16), ([5], [5], 2, 2, 96, 8), ([64], [64], 2, 1, 128, 16), ([65], [129], 2, 2, 128, 64), ([33, 1, 200], [40, 500, 200], 4, 2, 160, 32),
          ([128], [128], 1, 1, 256, 128), ([129], [1000], 8, 1, 64, 16), ([0, 7, 0, 90, 0], [10, 7, 0, 2000, 3], 6, 2, 32, 8), ([500], [500], 7, 1, 224, 16),
          ([17, 16, 15], [63, 64, 65], 3, 3, 192, 8), ([1000], [1023], 4, 4, 128, 1024)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(lc, shape, bits, dtype):
    new, lens, heads, kv, dim, page = shape
    run(lc, len(new) + dim, new, lens, heads, kv, dim, bits, dtype, page)


@pytest.mark.parametrize("dtype", TYPES)
def test_without_parts(lc, dtype):
    """Rows enough that no sequence is split along its tokens."""
    run(lc, 3, [300, 40, 1100], [900, 41, 1100], 32, 16, 64, 8, dtype, 16)


@pytest.mark.parametrize("dtype", TYPES)
def test_scales(lc, dtype):
    for scale in (0.0, -0.3, 2.0):
        run(lc, 4, [70], [200], 2, 1, 64, 8, dtype, 8, scale)


@pytest.mark.parametrize("dtype", TYPES)
def test_more_new_tokens_than_cached_ones(lc, dtype):
    """Those before the first cached token see nothing: zeros."""
    cache, table = filled(lc, 5, [20, 1], 2, 64, 8, 8)
    q = torch.randn(60, 4, 64, device=DEV).to(dtype)
    got = lc.lc_kv_attend_prompt(cache, q, ints([0, 50, 60]), table, ints([20, 0]))
    assert not got[:30].any() and not got[50:].any()
    check(got, *want_of(lc, cache, q, [0, 50, 60], table, [20, 0]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [8, 4])
def test_pages_that_are_not_there(lc, dtype, bits):
    """Pages outside the cache count as not seen, also where they are all a token would see; lengths beyond the table are held to it."""
    cache, table = filled(lc, 6, [100, 100], 1, 64, bits, 16)
    table[0, 0], table[0, 3], table[1] = -1, cache.pages, 2 ** 31 - 1
    lens = [100, 100]
    q = torch.randn(200, 2, 64, device=DEV).to(dtype)
    starts = [0, 100, 200]
    got = lc.lc_kv_attend_prompt(cache, q, ints(starts), table, ints(lens))
    assert not got[:16].any() and not got[100:].any()
    check(got, *want_of(lc, cache, q, starts, table, lens))
    cache, table = filled(lc, 6, [112], 1, 64, bits, 16)
    assert torch.equal(lc.lc_kv_attend_prompt(cache, q[:50], ints([0, 50]), table, ints([10 ** 9])), lc.lc_kv_attend_prompt(cache, q[:50], ints([0, 50]), table, ints([112])))
    assert not lc.lc_kv_attend_prompt(cache, q[:50], ints([0, 50]), table, ints([-7])).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [40, 300])
def test_what_is_not_finite(lc, dtype, new):
    """A key or value that is not finite gives NaN to the tokens that see it and to no others; a query with an infinity or NaN to itself."""
    for name in ("k", "v"):
        cache, table = filled(lc, 7, [new + 50], 1, 64, 8, 16)
        t = new + 50 - 13
        slot = int(table[0, t // 16]) * 16 + t % 16
        k, v = lc.lc_kv_read(cache, torch.tensor([slot], device=DEV))
        (k if name == "k" else v)[0, 0, 3] = float("inf")
        lc.lc_kv_write(cache, k, v, torch.tensor([slot], device=DEV))
        q = torch.randn(new, 3, 64, device=DEV).to(dtype)
        got = lc.lc_kv_attend_prompt(cache, q, ints([0, new]), table, ints([new + 50]))
        assert got[new - 13:].isnan().all() and got[:new - 13].isfinite().all()
        keep = [0, new - 13]
        check(got[:new - 13], *want_of(lc, cache, q[:new - 13], keep, table, [new + 50 - 13]))
    cache, table = filled(lc, 7, [new + 50], 1, 64, 8, 16)
    q = torch.randn(new, 3, 64, device=DEV).to(dtype)
    q[3, 1, 5], q[20, 0, 0], q[21, 2, 63] = float("inf"), float("nan"), -float("inf")
    got = lc.lc_kv_attend_prompt(cache, q, ints([0, new]), table, ints([new + 50]))
    nan = torch.zeros(new, 3, dtype=torch.bool, device=DEV)
    nan[3, 1] = nan[20, 0] = nan[21, 2] = True
    assert torch.equal(got.isnan().all(-1), nan) and torch.equal(got.isnan().any(-1), nan)


@pytest.mark.parametrize("dtype", TYPES)
def test_values_of_unlike_sizes(lc, dtype):
    """Scales of values from 2^-12 to 2^12 side by side, and scores far apart."""
    cache, table = filled(lc, 8, [400], 2, 128, 8, 16)
    g = torch.Generator(DEV).manual_seed(2)
    slots = torch.tensor([int(table[0, t // 16]) * 16 + t % 16 for t in range(400)], device=DEV)
    k, v = (torch.randn(400, 2, 128, device=DEV, generator=g) for _ in range(2))
    lc.lc_kv_write(cache, 4 * k, v * torch.exp2(torch.randint(-12, 13, (400, 2, 1), device=DEV, generator=g)), slots)
    q = (3 * torch.randn(150, 4, 128, device=DEV, generator=g)).to(dtype)
    check(lc.lc_kv_attend_prompt(cache, q, ints([0, 150]), table, ints([400])), *want_of(lc, cache, q, [0, 150], table, [400]))


def test_values_beyond_fp16(lc):
    """In fp16 only results have to fit."""
    cache = lc.new_kv_cache(1, 1, 8, 32, 8)
    v = torch.full((2, 1, 32), 1e5, device=DEV)
    v[1] = -3e4
    lc.lc_kv_write(cache, torch.zeros_like(v), v, torch.tensor([0, 1], device=DEV))
    q = torch.zeros(2, 1, 32, dtype=torch.float16, device=DEV)
    got = lc.lc_kv_attend_prompt(cache, q, ints([0, 2]), ints([[0]]), ints([2])).float()
    assert (got[0] == float("inf")).all() and ((got[1] - 3.5e4).abs() <= 16 + (1e5 + 3e4) / 2 * 2.0 ** -11).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("step", [-3, 3])
def test_values_that_grow_and_shrink(lc, dtype, step):
    """Scales of values by 2^3 a tile up or down, to 2^45; with an even probability over all, and one that follows the small ones: each row's result within its
    type's roundings of the values that carry it."""
    n = 960
    cache, table = filled(lc, 14, [n], 1, 64, 8, 16)
    g = torch.Generator(DEV).manual_seed(3)
    slots = torch.tensor([int(table[0, t // 16]) * 16 + t % 16 for t in range(n)], device=DEV)
    k, v = (torch.randn(n, 1, 64, device=DEV, generator=g) for _ in range(2))
    power = torch.arange(n, device=DEV) // 64 * step
    lc.lc_kv_write(cache, 0.1 * k, v * torch.exp2(power.float() - (0 if step < 0 else 45))[:, None, None], slots)
    q = torch.randn(n, 2, 64, device=DEV, generator=g).to(dtype)
    check(lc.lc_kv_attend_prompt(cache, q, ints([0, n]), table, ints([n])), *want_of(lc, cache, q, [0, n], table, [n]))


@pytest.mark.parametrize("dtype", TYPES)
def test_values_of_zero(lc, dtype):
    """Vectors of zeros, whose scale is zero, count in the sum of probabilities: first alone, then among others."""
    cache, table = filled(lc, 15, [200], 1, 64, 8, 16)
    slots = torch.tensor([int(table[0, t // 16]) * 16 + t % 16 for t in range(200)], device=DEV)
    k, v = (torch.randn(200, 1, 64, device=DEV) for _ in range(2))
    v[:100], k[30:60] = 0, 0
    v[::3] = 0
    lc.lc_kv_write(cache, k, v, slots)
    q = torch.randn(200, 1, 64, device=DEV).to(dtype)
    check(lc.lc_kv_attend_prompt(cache, q, ints([0, 200]), table, ints([200])), *want_of(lc, cache, q, [0, 200], table, [200]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv", [(4, 2), (64, 64)])
def test_rows_with_pitches_and_rows_of_no_sequence(lc, dtype, heads, kv):
    cache, table = filled(lc, 9, [30, 200], kv, 32, 8, 8)
    qkv = torch.randn(250, heads * 32 * 2 + 16, device=DEV).to(dtype)
    q = qkv[:, 16:16 + heads * 32].view(250, heads, 32)
    out = torch.full((250, heads * 32 + 8), 7.0, dtype=dtype, device=DEV)
    view = out[:, :heads * 32].view(250, heads, 32)
    starts = [5, 25, 225]
    lc.lc_kv_attend_prompt(cache, q, ints(starts), table, ints([30, 200]), out=view)
    assert (out[:5] == 7).all() and (out[225:] == 7).all() and (out[:, heads * 32:] == 7).all()
    want, room = want_of(lc, cache, q, starts, table, [30, 200])
    check(view[5:225], want[5:225], room[5:225])


@pytest.mark.parametrize("dtype", TYPES)
def test_the_same_as_drafted_tokens_one_after_the_other(lc, dtype):
    """lc_kv_attend and this one within both their roundings of each other."""
    cache, table = filled(lc, 10, [90, 90, 90], 2, 128, 8, 16)
    q = torch.randn(3, 64, 4, 128, device=DEV).to(dtype)
    a = lc.lc_kv_attend(cache, q, table, ints([90] * 3))
    starts = [0, 64, 128, 192]
    b = lc.lc_kv_attend_prompt(cache, q.view(192, 4, 128), ints(starts), table, ints([90] * 3))
    want, room = want_of(lc, cache, q.view(192, 4, 128), starts, table, [90] * 3)
    check(b, want, room)
    check(a.view(192, 4, 128), want, room)


def test_many_sequences(lc):
    """More sequences than a wavefront has lanes, most of one new token."""
    new = [1 + (b % 7 == 0) * (b % 40) for b in range(150)]
    lens = [n + (b * 13) % 90 for b, n in enumerate(new)]
    run(lc, 11, new, lens, 4, 2, 64, 8, torch.bfloat16, 8)


@pytest.mark.parametrize("dtype", TYPES)
def test_more_than_64_sequences_some_of_them_split(lc, dtype):
    """One long one among many short ones, empty ones among them, in any order; and 64 and 65 of them."""
    for batch, heads, kv in ((70, 4, 2), (64, 2, 2), (65, 2, 2), (1100, 2, 1)):
        new = [(b * 7) % 5 for b in range(batch)]
        lens = [max(1, n + (b * 11) % 40) for b, n in enumerate(new)]
        new[batch // 2], lens[batch // 2] = 100, 1500
        new[3], lens[3] = 40, 900
        run(lc, batch, new, lens, heads, kv, 32, 8, dtype, 8)


def test_as_many_sequences_as_there_may_be(lc):
    """65535 of a token each, all over one page, and of none: the same as one alone."""
    cache, table = filled(lc, 16, [8], 1, 32, 8, 8)
    q = torch.randn(1, 2, 32, device=DEV).to(torch.bfloat16)
    want = lc.lc_kv_attend_prompt(cache, q, ints([0, 1]), table, ints([5]))
    n = 65535
    got = lc.lc_kv_attend_prompt(cache, q.expand(n, 2, 32).contiguous(), torch.arange(n + 1, dtype=torch.int32, device=DEV), table.expand(n, 1).contiguous(),
                                 torch.full((n,), 5, dtype=torch.int32, device=DEV))
    assert torch.equal(got, want.expand(n, 2, 32))
    starts = torch.ones(n + 1, dtype=torch.int32, device=DEV)
    starts[:30000] = 0
    assert torch.equal(lc.lc_kv_attend_prompt(cache, q, starts, table.expand(n, 1).contiguous(), torch.full((n,), 5, dtype=torch.int32, device=DEV)), want)


def test_a_long_cache(lc):
    """Codes beyond 4 GiB from where they begin."""
    pages, kv, page, dim = 9000, 8, 512, 128
    cache = lc.KvCache(torch.empty(pages, kv, page, dim, dtype=torch.uint8, device=DEV), torch.empty(pages, kv, page, dim, dtype=torch.uint8, device=DEV),
                       torch.zeros(pages, kv, page, device=DEV), torch.zeros(pages, kv, page, device=DEV), 8)
    assert cache.k.numel() > 1 << 32
    slots = torch.tensor([8999 * page + t for t in range(300)], device=DEV)
    k, v = torch.randn(300, kv, dim, device=DEV), torch.randn(300, kv, dim, device=DEV)
    lc.lc_kv_write(cache, k, v, slots)
    q = torch.randn(100, kv, dim, device=DEV).to(torch.bfloat16)
    table = ints([[8999]])
    check(lc.lc_kv_attend_prompt(cache, q, ints([0, 100]), table, ints([300])), *want_of(lc, cache, q, [0, 100], table, [300]))


def test_on_another_stream_and_in_a_graph(lc):
    for heads, kv in ((4, 2), (64, 32)):
        lens = [300, 64]
        cache, table = filled(lc, 12, lens, kv, 64, 8, 16)
        q = torch.randn(164, heads, 64, device=DEV).to(torch.bfloat16)
        starts = ints([0, 100, 164])
        want = lc.lc_kv_attend_prompt(cache, q, starts, table, ints(lens))
        s = torch.cuda.Stream()
        n = ints(lens)
        s.wait_stream(torch.cuda.current_stream())
        got = lc.lc_kv_attend_prompt(cache, q, starts, table, n, stream=s)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(got, want)
        ws, out = lc.new_prompt_workspace(cache, 164, 2, heads), torch.empty_like(q)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lc.lc_kv_attend_prompt(cache, q, starts, table, n, out=out, ws=ws)
        for i in range(3):
            q.copy_(torch.randn(q.shape, device=DEV))
            n.copy_(ints([300 - 100 * i, 64 - i]))
            graph.replay()
            got = out.clone()
            ws.fill_(255)
            assert torch.equal(got, lc.lc_kv_attend_prompt(cache, q, starts, table, n))


def test_nothing_new(lc):
    cache, table = filled(lc, 13, [10], 1, 32, 8, 8)
    assert lc.lc_kv_attend_prompt(cache, torch.empty(0, 1, 32, device=DEV), ints([0, 0]), table, ints([10])).shape == (0, 1, 32)
    out = torch.full((4, 1, 32), 5.0, device=DEV)
    lc.lc_kv_attend_prompt(cache, torch.randn(4, 1, 32, device=DEV), ints([2, 2]), table, ints([10]), out=out)
    assert (out == 5).all()
    empty = torch.empty(0, 1, 8, 32, dtype=torch.uint8, device=DEV)
    none = torch.empty(0, 1, 8, device=DEV)
    got = lc.lc_kv_attend_prompt(lc.KvCache(empty, empty.clone(), none, none.clone(), 8), torch.randn(4, 1, 32, device=DEV), ints([0, 4]), ints([[0]]), ints([8]))
    assert not got.any()


def test_refused(lc):
    cache, table = filled(lc, 13, [10], 2, 32, 8, 8)
    q = torch.randn(4, 2, 32, device=DEV)
    with pytest.raises(AssertionError):
        lc.lc_kv_attend_prompt(cache, q.requires_grad_(), ints([0, 4]), table, ints([10]))
    q = q.detach()
    with pytest.raises(AssertionError):
        lc.lc_kv_attend_prompt(cache, q, ints([0, 4, 4]), table, ints([10]))
    with pytest.raises(lc.LcError):
        lc.lc_kv_attend_prompt(cache, torch.randn(4, 3, 32, device=DEV), ints([0, 4]), table, ints([10]))
    with pytest.raises(lc.LcError):
        lc.lc_kv_attend_prompt(cache, q, ints([0, 4]), table, ints([10]), ws=torch.empty(0, dtype=torch.uint8, device=DEV))
