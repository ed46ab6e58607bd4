"""Attention of many new tokens a sequence, with more workgroups than one launch has room for: 65535 sequences over a cache of 256 heads are 2^24 of them, 2^32 threads or more."""
import pytest
import torch

from .test_gpu_prompt import DEV, ints

pytestmark = pytest.mark.gpu


def test_many_sequences_over_many_heads():
    from paper_2009_13003_amd import lc
    heads, n, page = 256, 65535, 8
    cache = lc.new_kv_cache(7, heads, page, 32, 8)
    g = torch.Generator(DEV).manual_seed(1)
    k, v = (torch.randn(7 * page, heads, 32, device=DEV, generator=g) for _ in range(2))
    lc.lc_kv_write(cache, k, v, torch.arange(7 * page, device=DEV))
    few = torch.randn(63, heads, 32, device=DEV, generator=g).to(torch.bfloat16)
    q = few.repeat(n // 63 + 1, 1, 1)[:n]
    number = torch.arange(n, dtype=torch.int32, device=DEV)
    table, lens = (number % 7).view(n, 1), number % 9        # (0: sees nothing)
    out = lc.lc_kv_attend_prompt(cache, q, torch.arange(n + 1, dtype=torch.int32, device=DEV), table, lens)
    want = lc.lc_kv_attend_prompt(cache, few, ints(list(range(64))), table[:63].contiguous(), lens[:63])       # (63 sequences, and so all of them again and again)
    whole = n // 63 * 63
    assert (out[:whole].view(-1, 63, heads, 32) == want).all() and torch.equal(out[whole:], want[:n - whole])
    assert not out[::9].any() and out[1::9].any(-1).all()
