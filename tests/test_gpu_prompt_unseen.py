"""Attention of many new tokens a sequence: what is not seen does not matter, whatever it holds.  Scales that nobody sees are numbers here, and large ones, next to what is seen."""
import pytest
import torch

from .test_gpu_prompt import DEV, TYPES, check, filled, ints, want_of

pytestmark = pytest.mark.gpu
FILLS = [1.0, 2.0 ** 30, 1e30, 3e38, -1e30]                  # beside scales of some 0.02 that are seen


@pytest.fixture(scope="module")
def lc():
    from paper_2009_13003_amd import lc
    return lc


def queries(tokens, heads, dim, dtype, seed=1):
    return (1.5 * torch.randn(tokens, heads, dim, device=DEV, generator=torch.Generator(DEV).manual_seed(seed))).to(dtype)


def starts_of(new):
    s = [0]
    for n in new:
        s.append(s[-1] + n)
    return s


def same_whatever_is_not_seen(lc, cache, unseen, q, starts, table, lens):
    """Results with zeros in the scales that nobody sees: within their room, and the same bits with any other numbers there."""
    def put(v):
        cache.k_scale[unseen], cache.v_scale[unseen] = v, v
    put(0.0)
    want = lc.lc_kv_attend_prompt(cache, q, ints(starts), table, ints(lens))
    check(want, *want_of(lc, cache, q, starts, table, lens))
    for v in FILLS:
        put(v)
        got = lc.lc_kv_attend_prompt(cache, q, ints(starts), table, ints(lens))
        assert torch.equal(got, want), (v, (got.float() - want.float()).abs().max().item(), want.float().abs().max().item())


# new tokens, cached ones, heads, heads of the cache, elements, page: one tile and several, lengths that are no multiple of 8, split along the tokens or not
BEHIND = [([1], [1], 1, 1, 32, 8), ([60], [60], 2, 1, 64, 16), ([1], [300], 4, 2, 64, 16), ([100], [100], 16, 16, 64, 16), ([9], [2001], 2, 1, 128, 64), ([17, 16, 15], [63, 66, 65], 3, 3, 96, 8),
          ([33, 1, 200], [45, 500, 207], 4, 2, 160, 32), ([130], [131], 1, 1, 256, 128), ([300, 40, 1101], [900, 41, 1101], 32, 16, 64, 16)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("shape", BEHIND, ids=str)
def test_places_behind_the_last_token(lc, shape, bits, dtype):
    new, lens, heads, kv, dim, page = shape
    cache, table = filled(lc, 20 + dim, lens, kv, dim, bits, page)
    same_whatever_is_not_seen(lc, cache, cache.v_scale.isnan(), queries(sum(new), heads, dim, dtype), starts_of(new), table, lens)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,lens,page", [([70], [100], 16), ([40, 130], [1000, 140], 8), ([100], [190], 64)], ids=str)
def test_pages_that_are_not_there(lc, new, lens, page, bits, dtype):
    """Another page is read in their place: none that anybody sees here."""
    cache, table = filled(lc, 31, lens, 2, 64, bits, page)
    unseen = cache.v_scale.isnan()
    found = (table == 0).nonzero().tolist()
    assert len(found) <= 1
    for b, j in found:                                       # (the page that stands in for others)
        table[b, j] = -1
    unseen[0] = True
    table[0, 0], table[-1, -(-lens[-1] // page) - 1] = cache.pages, 2 ** 31 - 1
    same_whatever_is_not_seen(lc, cache, unseen, queries(sum(new), 4, 64, dtype), starts_of(new), table, lens)


def later_ones_larger(lc, seed, n, kv, dim, bits, page, power):
    """A cache of one sequence of n tokens, of which number t has values of a size of 2^power[t]."""
    cache, table = filled(lc, seed, [n], kv, dim, bits, page)
    g = torch.Generator(DEV).manual_seed(seed)
    k, v = (torch.randn(n, kv, dim, device=DEV, generator=g) for _ in range(2))
    slots = torch.tensor([int(table[0, t // page]) * page + t % page for t in range(n)], device=DEV)
    lc.lc_kv_write(cache, k, v * torch.exp2(torch.as_tensor(power, dtype=torch.float32, device=DEV))[:, None, None], slots)
    return cache, table


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("power", [24, 40, 80])
@pytest.mark.parametrize("new,n,heads,kv,first", [(300, 300, 1, 1, 200), (300, 300, 2, 2, 128), (64, 64, 1, 1, 20), (40, 2000, 2, 1, 1985), (600, 1000, 8, 2, 770)])
def test_later_blocks_of_rows(lc, new, n, heads, kv, first, power, dtype):
    """Tokens from `first` on have values 2^power times as large.  Those before are within the room that what they see gives them."""
    cache, table = later_ones_larger(lc, 40 + new, n, kv, 64, 8, 16, [power * (t >= first) for t in range(n)])
    q = queries(new, heads, 64, dtype)
    got = lc.lc_kv_attend_prompt(cache, q, ints([0, new]), table, ints([n]))
    few = first - (n - new)
    want, room = want_of(lc, cache, q[:few], [0, few], table, [first])
    # (a score measured from up to 2^7 away is rounded to 2^-18 at most, in the products and in their sum: 2^-17 ln 2 of the result's products, whose own
    # rounding to 2^-11 is in the room; fp32 does not measure so)
    check(got[:few], want, room * (1 if dtype == torch.float32 else 1 + 2.0 ** -6))
    if dtype != torch.float16:
        check(got[few:], *(t[few:] for t in want_of(lc, cache, q, [0, new], table, [n])))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,cached", [(64, 64), (90, 90), (70, 1000)])
def test_every_token_larger_than_the_one_before(lc, n, cached, dtype):
    """Values that double from token to token over the new ones: each one's room is that of what it sees."""
    base = cached - n
    cache, table = later_ones_larger(lc, 50 + n, cached, 1, 64, 8, 16, [max(0, t - base) - 40 for t in range(cached)])
    q = queries(n, 2, 64, dtype)
    got = lc.lc_kv_attend_prompt(cache, q, ints([0, n]), table, ints([cached]))
    for i in list(range(0, n, 5)) + [n - 1]:
        want, room = want_of(lc, cache, q[i:i + 1], [0, 1], table, [base + i + 1])
        check(got[i:i + 1], want, room * (1 if dtype == torch.float32 else 1 + 2.0 ** -6))
