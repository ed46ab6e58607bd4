"""Products with infinities and NaN against the same product without: the ratio of the two times on one card, the fastest of many calls each.
The bounds lie midway (by ratio) between what such inputs took element by element (430, 160 and 16 times the product) and what they take now (1.5, 1.2 and 4.4)."""
import pytest
import torch

from tests.test_gpu_relative_times import best_us

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_times_of_what_is_not_finite(dtype):
    from paper_2009_13003_amd import lc
    g = torch.Generator(device=DEV); g.manual_seed(1)
    w4 = lc.lc_w4_quantize(torch.randn(4096, 4096, generator=g, device=DEV), 128)
    x = torch.randn(256, 4096, generator=g, device=DEV).to(dtype)
    plain = best_us(lambda: lc.lc_w4_matmul(x, w4), 20)
    nan, one = torch.full_like(x, float("nan")), x.clone()
    one[0, 0] = float("inf")
    assert lc.lc_w4_matmul(nan, w4).isnan().all()
    assert best_us(lambda: lc.lc_w4_matmul(nan, w4), 20) <= 25 * plain
    y = lc.lc_w4_matmul(one, w4)
    q = (w4.codes[:, 0] & 15).int() - 8                      # what the infinity is multiplied by
    assert ((y[0] == float("inf")) == (q > 0)).all() and ((y[0] == -float("inf")) == (q < 0)).all() and (y[0].isnan() == (q == 0)).all()
    assert torch.equal(y[1:], lc.lc_w4_matmul(x, w4)[1:])
    assert best_us(lambda: lc.lc_w4_matmul(one, w4), 20) <= 8.5 * plain
    w4.scales[5, -1] = float("nan")
    y = lc.lc_w4_matmul(x, w4)
    assert y[:, 5].isnan().all() and not y[:, :5].isnan().any() and not y[:, 6:].isnan().any()
    assert best_us(lambda: lc.lc_w4_matmul(x, w4), 20) <= 14 * plain
