"""Products of as many results as no single launch has threads for."""
import pytest
import torch

from tests.test_gpu_w4 import check, random_w4

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lc():
    from paper_2009_13003_amd import lc as mod
    return mod


@pytest.mark.parametrize("bias", [True, False])
def test_no_width_and_two_to_the_32_results(lc, bias):
    m, n = 1 << 19, 8192 + 3                                 # 8 GiB
    w4 = lc.lc_w4_quantize(torch.zeros(n, 0, device=DEV), 32)
    b = torch.arange(n, device=DEV).remainder(100).to(torch.bfloat16) if bias else None
    out = torch.full((m, n), 7.0, dtype=torch.bfloat16, device=DEV)
    lc.lc_w4_matmul(torch.zeros(m, 0, dtype=torch.bfloat16, device=DEV), w4, b, out=out)
    want = b if bias else torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    for i in range(0, m, 1 << 14):
        assert torch.equal(out[i:i + (1 << 14)], want.expand(1 << 14, n))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [(1 << 17) - 128, (1 << 17) - 127, 2 * ((1 << 17) - 128) + 1])
def test_rows_of_w_in_several_launches(lc, dtype, n):
    g = torch.Generator(device=DEV); g.manual_seed(n)
    w4 = random_w4(lc, n, 40, 32, n)
    x, bias = torch.randn(40, 40, generator=g, device=DEV).to(dtype), torch.randn(n, generator=g, device=DEV).to(dtype)
    check(x, w4, bias, lc.lc_w4_matmul(x, w4, bias))
