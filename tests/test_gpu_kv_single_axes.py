"""Keys and values whose pitches differ only along an axis of one element are laid out alike: that pitch says nothing."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("tokens,heads", [(1, 3), (5, 1), (1, 1)])
def test_pitches_of_single_elements(tokens, heads):
    from paper_2009_13003_amd import lc
    cache, other = (lc.new_kv_cache(2, heads, 8, 32, 8, DEV) for _ in range(2))
    g = torch.Generator(device=DEV); g.manual_seed(3)
    k = torch.randn(tokens, heads, 32, generator=g, device=DEV)
    store = torch.full((tokens, heads, 64), 9.0, device=DEV)
    # the same pitches where there is more than one, others where there is not
    v = torch.as_strided(store, (tokens, heads, 32), (heads * 32 if tokens > 1 else 7, 32 if heads > 1 else 5, 1))
    v.copy_(torch.randn(tokens, heads, 32, generator=g, device=DEV))
    slots = torch.arange(tokens, device=DEV) + 2
    lc.lc_kv_write(cache, k, v, slots)
    lc.lc_kv_write(other, k, v.contiguous().clone(), slots)
    assert torch.equal(cache.v, other.v) and torch.equal(cache.v_scale, other.v_scale) and torch.equal(cache.k, other.k)
    want = lc.lc_kv_read(cache, slots)
    got = torch.empty_like(k), v
    lc.lc_kv_read(cache, slots, out=got)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
