"""The serving operators have no backward pass: on tensors that a gradient is asked for they refuse, instead of giving results that none flows
through."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_gradients_are_refused():
    from paper_2009_13003_amd import lc
    w = torch.randn(32, 64, device=DEV, requires_grad=True)
    w4 = lc.lc_w4_quantize(w, 32)                            # what is stored has no gradient: parameters as they are
    x, bias = torch.randn(3, 64, device=DEV), torch.randn(32, device=DEV)
    cache = lc.new_kv_cache(2, 1, 8, 32, 8, DEV)
    k, slots = torch.randn(3, 1, 32, device=DEV), torch.arange(3, device=DEV)
    table, lens = torch.tensor([[0, 1]], dtype=torch.int32, device=DEV), torch.tensor([3], dtype=torch.int32, device=DEV)
    q = torch.randn(1, 1, 1, 32, device=DEV)
    calls = [lambda t: lc.lc_w4_matmul(t(x), w4), lambda t: lc.lc_w4_matmul(x, w4, t(bias)), lambda t: lc.lc_kv_write(cache, t(k), k, slots),
             lambda t: lc.lc_kv_write(cache, k, t(k), slots), lambda t: lc.lc_kv_attend(cache, t(q), table, lens)]
    for call in calls:
        with pytest.raises(AssertionError, match="gradient"):
            call(lambda v: v.clone().requires_grad_())
    for call in calls:
        want = call(lambda v: v)
        with torch.no_grad():
            got = call(lambda v: v.clone().requires_grad_())
        with torch.inference_mode():
            also = call(lambda v: v.clone())
        assert want is None or (torch.equal(got, want) and torch.equal(also, want) and not got.requires_grad)
