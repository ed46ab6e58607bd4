"""Scratch for attention of many new tokens a sequence: an area of lc_kv_prompt_workspace_most is enough for every call of up to its sizes (no GPU needed)."""
import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2009_13003_amd import lc
    return lc._lib


TOKENS = [0, 1, 2, 31, 128, 511, 1024, 2047, 2048, 4095, 4096, 16383, 16384, 100000, 1 << 18]
BATCH = [0, 1, 2, 9, 64, 65, 1000, 65535]


@pytest.mark.parametrize("heads,kv,dim", [(32, 8, 128), (32, 32, 128), (12, 4, 96), (1, 1, 32), (16, 16, 64), (9, 3, 256), (7, 7, 160), (300, 300, 64), (600, 600, 32), (4096, 1024, 32),
                                          (4096, 1, 64)])
def test_enough_for_every_smaller_call(lib, heads, kv, dim):
    need, most = lib.lc_kv_prompt_workspace_bytes, lib.lc_kv_prompt_workspace_most
    for i, tokens in enumerate(TOKENS):
        for j, batch in enumerate(BATCH):
            area = most(tokens, batch, heads, kv, dim)
            assert area >= 256 and area % 256 == 0
            for t in TOKENS[:i + 1]:
                for b in BATCH[:j + 1]:
                    assert need(t, b, heads, kv, dim) <= area, (tokens, batch, t, b)


def test_sizes_that_are_not_taken(lib):
    for bad in (((1 << 24) + 1, 1, 1, 1, 64), (1, 65536, 1, 1, 64), (1, 1, 3, 2, 64), (1, 1, 0, 1, 64), (1, 1, 4097, 1, 64), (1, 1, 1, 1, 48), (1 << 20, 1, 2048, 1024, 32)):
        assert lib.lc_kv_prompt_workspace_most(*bad) == 0


@pytest.mark.gpu
def test_one_area_for_prompts_of_any_length():
    """Made for the longest, whose rows need no splitting, and used for shorter ones, whose do."""
    import torch
    from paper_2009_13003_amd import lc
    g = torch.Generator("cuda").manual_seed(1)
    cache = lc.new_kv_cache(313, 8, 16, 128, 8)
    k, v = (torch.randn(313 * 16, 8, 128, device="cuda", generator=g) for _ in range(2))
    lc.lc_kv_write(cache, k, v, torch.arange(313 * 16, device="cuda"))
    table = torch.arange(313, dtype=torch.int32, device="cuda").view(1, 313)
    ws = lc.new_prompt_workspace(cache, 2048, 1, 32)
    for n in (2048, 2047, 513, 64, 1):
        q = torch.randn(n, 32, 128, device="cuda", generator=g).to(torch.bfloat16)
        starts, lens = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([0, n], [5000]))
        ws.fill_(255)
        assert torch.equal(lc.lc_kv_attend_prompt(cache, q, starts, table, lens, ws=ws), lc.lc_kv_attend_prompt(cache, q, starts, table, lens))
