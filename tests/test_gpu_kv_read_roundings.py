"""Reading the cache back: each value is the product of code and scale rounded to fp32, and that rounded to the type.  One rounding in place of the two
gives something else where the first ends halfway between two numbers of the type, so every code meets many scales."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [8, 4])
def test_two_roundings(dtype, bits):
    from paper_2009_13003_amd import lc
    pages, heads, page = 64, 4, 128
    dim = 256 if bits == 8 else 32
    g = torch.Generator(device=DEV); g.manual_seed(bits)
    scales = torch.exp2(8 * torch.rand(2, pages, heads, page, generator=g, device=DEV) - 6)
    row = torch.arange(256, device=DEV) if bits == 8 else torch.arange(16, device=DEV) * 17          # every byte; every nibble twice
    codes = row.to(torch.uint8).expand(pages, heads, page, row.numel()).contiguous()
    cache = lc.KvCache(codes, codes.clone(), scales[0], scales[1], bits)
    got = lc.lc_kv_read(cache, torch.arange(pages * page, device=DEV), dtype)
    q = row.cpu().numpy().astype(np.uint8).view(np.int8).astype(np.float32) if bits == 8 else np.repeat(np.arange(16), 2).astype(np.float32) - 8
    for n in range(2):
        s = scales[n].transpose(1, 2).reshape(-1, heads, 1).cpu().numpy()
        want = torch.from_numpy(q * s).to(dtype)             # (numpy's product of fp32 is rounded to fp32)
        assert want.shape == (pages * page, heads, dim) and torch.equal(got[n].cpu(), want)
