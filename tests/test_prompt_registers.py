"""Registers of the prompts' kernels with one wavefront a SIMD, as built: fp32, and 16 bits from 160 elements on.  Only fp32 heads of 256 put some away, as many as when they were measured."""
import os

import pytest

from .test_kernel_resources import ROCM, registers_of


@pytest.mark.skipif(not os.path.exists(os.path.join(ROCM, "llvm", "bin", "llvm-readelf")), reason="needs llvm-readelf")
def test_registers_of_the_library_as_built(tmp_path):
    from paper_2009_13003_amd import build
    if not os.path.exists(build.LIB):
        build.build_library()
    found = registers_of(build.LIB, tmp_path)
    for t in range(3):
        for bits in (8, 4):
            for dim in range(32 if t == 0 else 160, 257, 32):
                match = [v for k, v in found.items() if "11k_kv_promptILi%dELi%dELi%dELi4ELi1E" % (t, bits, dim) in k]
                assert len(match) == 1 and match[0][0] <= 512 and match[0][1] <= (170 if (t, dim) == (0, 256) else 0), (t, bits, dim, match)
