"""Registers of the kernels of 8-bit products and prompts as built, on which the workgroups that share a compute unit, and so their measured times, depend."""
import os

import pytest

from .test_kernel_resources import ROCM, registers_of

# kernel (mangled name contains): vector registers at most, spilled ones at most.  Prompts in 16 bits up to 128 elements: two wavefronts a SIMD; tiles of 8-bit products in
# workgroups of four wavefronts, one a SIMD (two of 64 x 64 and 128 x 64).
LIMITS = {"11k_kv_promptILi%dELi%dELi%dELi%dELi2E" % (t, bits, dim, waves): (256, 0) for t in (1, 2) for bits in (8, 4) for dim in (32, 64, 96, 128) for waves in (4, 8)}
LIMITS.update({"10k_i8_tilesILi128ELi256E": (512, 0), "10k_i8_tilesILi128ELi128E": (512, 0), "10k_i8_tilesILi128ELi64E": (256, 0), "10k_i8_tilesILi64ELi64E": (256, 0),
               "9k_i8_rowsILi1E": (64, 0), "9k_i8_rowsILi2E": (72, 0)})
LIMITS.update({"12k_i8_one_rowILi%dELi%dE" % (t, r): (84 if r == 1 else 128, 0) for t in range(3) for r in (1, 3)})
LIMITS.update({"15k_i8_short_rowsILi%dELi%dE" % (t, r): (84, 0) for t in range(3) for r in (1, 2)})


@pytest.mark.skipif(not os.path.exists(os.path.join(ROCM, "llvm", "bin", "llvm-readelf")), reason="needs llvm-readelf")
def test_registers_of_the_library_as_built(tmp_path):
    from paper_2009_13003_amd import build
    if not os.path.exists(build.LIB):
        build.build_library()
    found = registers_of(build.LIB, tmp_path)
    for name, (registers, spills) in LIMITS.items():
        match = [v for k, v in found.items() if name in k]
        assert len(match) == 1, (name, sorted(found))
        assert match[0][0] <= registers and match[0][1] <= spills, (name, match)
