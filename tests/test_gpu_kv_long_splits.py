"""Attention over the cache where sequences are split into parts of several units of 128 tokens, into as many parts as there may be, and where the
search for a part's sequence passes the first 64 sequences: against 64 bits, with test_gpu_kv's bounds."""
import pytest
import torch

from tests.test_gpu_kv import Case, tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lc():
    from paper_2009_13003_amd import lc as mod
    return mod


MANY = [0 if i % 9 == 4 else 3000 + i if i % 31 == 7 else 1 + i * 37 % 700 for i in range(100)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("lens,nq,heads,kv,dim,page", [
    ([8191, 6552, 4914, 3276, 1638], 24, 32, 8, 128, 32),    # parts of 11 units: the first length tried gives too many of them
    ([8500], 1, 4, 1, 64, 16),                               # more units than the 60 parts that a sequence may have
    ([20000, 10, 0], 1, 2, 1, 128, 64),                      # ... where the slots alone would allow more
    (MANY, 1, 1, 1, 64, 8),                                  # sequences beyond the first 64, some of them empty, some in many parts
    (MANY[:70], 3, 2, 2, 96, 16)])
def test_long_and_many(lc, dtype, bits, lens, nq, heads, kv, dim, page):
    case = Case(lc, sum(lens) + nq, lens, nq, heads, kv, dim, page, bits, dtype)
    mask = tree(len(lens), nq, nq) if nq > 1 else None
    case.check(case.run(lc, mask), mask)
