"""A query with an infinity: whatever it sees has a score that is infinite or no number, so all of its result is NaN, and zeros where it sees
nothing."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dim", [64, 128, 160])
@pytest.mark.parametrize("tokens,nq", [(5, 1), (90, 20), (2000, 3)])
@pytest.mark.parametrize("sign", [1, -1])
def test_infinite_queries(dtype, bits, dim, tokens, nq, sign):
    from paper_2009_13003_amd import lc
    page = 16
    pages = -(-tokens // page)
    cache = lc.new_kv_cache(pages, 1, page, dim, bits, DEV)
    g = torch.Generator(device=DEV); g.manual_seed(dim + tokens)
    k = 0.5 + torch.rand(tokens, 1, dim, generator=g, device=DEV)        # above zero, in codes too: an infinity keeps its sign in every score
    lc.lc_kv_write(cache, k, torch.randn(tokens, 1, dim, generator=g, device=DEV), torch.arange(tokens, device=DEV))
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None]
    lens = torch.tensor([tokens], dtype=torch.int32, device=DEV)
    q = torch.randn(1, nq, 2, dim, generator=g, device=DEV).to(dtype)
    want = lc.lc_kv_attend(cache, q, table, lens)
    assert want.isfinite().all()
    for at in (0, dim // 2 + 5, dim - 1):
        bad = q.clone()
        bad[0, nq - 1, 1, at] = sign * float("inf")
        out = lc.lc_kv_attend(cache, bad, table, lens)
        assert out[0, nq - 1, 1].isnan().all()
        # the others as before, but for when their sums are rescaled: probabilities in 16 bits of values below 6, and the result's rounding
        both = torch.ones(nq, 2, dtype=torch.bool, device=DEV)
        both[nq - 1, 1] = False
        a, b = out[0][both].double(), want[0][both].double()
        assert ((a - b).abs() <= 2 * (6 * 2.0 ** -15 + HALF_ULP[dtype] * b.abs())).all()
    # sees none of the drafted tokens, of which there are more than cached ones: nothing at all
    lens.fill_(min(nq, tokens))
    out = lc.lc_kv_attend(cache, bad, table, lens, mask=torch.zeros(1, nq, dtype=torch.int64, device=DEV))
    assert (out == 0).all()
