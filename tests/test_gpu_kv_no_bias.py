"""Attention of 16-bit types keeps its probabilities with 16 bits and more, and loses nothing on average.  All values of a head are one number, 3e-6 beyond the middle
between two of the type, so that results have to be the upper one: probabilities that are cut off, 7e-6 too small on average, give the lower.

Each of about 1000 probabilities of like size is off by at most 2^-16 of itself, either way: together by 2^-16 / sqrt(3 * 1000) = 3e-7, a tenth of what is left; sums in
32 bits of a thousand positive numbers in tens of parts add as much again."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype,half", [(torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("nq,heads,dim", [(1, 4, 64), (1, 2, 128), (40, 4, 128), (2, 2, 256)])
def test_one_value(dtype, half, bits, nq, heads, dim):
    from paper_2009_13003_amd import lc
    page, tokens = 64, 1000
    pages, most = -(-tokens // page), 127 if bits == 8 else 7
    g = torch.Generator(device=DEV); g.manual_seed(dim + nq)
    cache = lc.new_kv_cache(pages, 2, page, dim, bits, DEV)
    k = torch.randn(pages * page, 2, dim, generator=g, device=DEV)
    lc.lc_kv_write(cache, k, torch.ones_like(k), torch.arange(pages * page, device=DEV))
    cache.v_scale.fill_((1 + half + 3e-6) / most)            # the codes of 1 are the largest
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None]
    q = (0.5 * torch.randn(1, nq, heads, dim, generator=g, device=DEV)).to(dtype)
    out = lc.lc_kv_attend(cache, q, table, torch.tensor([tokens], dtype=torch.int32, device=DEV))
    assert (out == 1 + 2 * half).all()
