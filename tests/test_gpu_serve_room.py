"""The decoder where shared pages hold what is written but not a tree of drafts beside it."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PROMPTS, COUNT = (28, 12, 44), 20                          # ends at the ends of pages
PAGES = sum(-(-(n + COUNT) // 16) for n in PROMPTS)          # of 16 tokens: what is known at the end, to the token


@pytest.fixture(scope="module")
def parts():
    from paper_2009_13003_amd import serve
    shape = serve.Shape(vocab=200, width=128, layers=2, heads=4, kv_heads=2, inner=96, context=300)
    g = torch.Generator(DEV).manual_seed(4)
    flat = 0.1 * torch.randn(shape.numel(), device=DEV, generator=g)
    return serve, shape, flat, [torch.randint(200, (n,), device=DEV, generator=g).tolist() for n in PROMPTS]


@pytest.mark.parametrize("drafts", [1, 2, 7])
def test_tokens_without_room_for_a_tree(parts, drafts):
    serve, shape, flat, prompts = parts
    want, _ = serve.write_on(serve.Decoder(shape, flat, 3, dtype=torch.float32, shared=60), prompts, COUNT, drafts)
    model = serve.Decoder(shape, flat, 3, dtype=torch.float32, shared=PAGES)
    got, passes = serve.write_on(model, prompts, COUNT, drafts)
    assert got == want and passes <= COUNT
    assert model.lens.tolist() == model.count == [n + COUNT - 1 for n in PROMPTS]
    drawn, _ = serve.write_on(serve.Decoder(shape, flat, 3, weights=8, shared=PAGES), prompts, COUNT, drafts, sample=torch.Generator(DEV).manual_seed(5))
    assert all(len(t) == COUNT and all(0 <= x < 200 for x in t) for t in drawn)


def test_no_room_for_the_tokens_themselves(parts):
    serve, shape, flat, prompts = parts
    for drafts in (0, 2):
        model = serve.Decoder(shape, flat, 3, dtype=torch.float32, shared=PAGES - 1)
        with pytest.raises(ValueError, match="shared pages"):
            serve.write_on(model, prompts, COUNT, drafts)
