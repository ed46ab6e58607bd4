"""Writing on up to the end of the context: where a tree of drafted tokens has no room any more, the last tokens are judged one at a time."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("drafts", [1, 2, 5])
@pytest.mark.parametrize("left", [0, 1, 4])
def test_up_to_the_end_of_the_context(drafts, left):
    from paper_2009_13003_amd import serve
    shape = serve.Shape(vocab=100, width=64, layers=1, heads=2, kv_heads=1, inner=64, context=60)
    g = torch.Generator(DEV).manual_seed(7)
    flat = 0.2 * torch.randn(shape.numel(), device=DEV, generator=g)
    prompt = torch.randint(100, (2, 40), device=DEV, generator=g)
    make = lambda: serve.Decoder(shape, flat, 2, 8, 32, torch.float32)
    alone, passes = serve.write_on(make(), prompt, 20 - left, drafts=0)
    assert passes == 20 - left and all(len(t) == 20 - left for t in alone)
    drafted, _ = serve.write_on(make(), prompt, 20 - left, drafts=drafts)
    assert drafted == alone
