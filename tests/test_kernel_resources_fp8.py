"""Register budgets of the kernels of training in 8 bits (see test_kernel_resources.py): two workgroups of 128 x 128 tiles and
four of 64 x 64 on a compute unit, nothing spilled; the 256 x 256 ones take all registers, and what spills is a few values of
the last rows on their way out."""
import os
import re

import pytest

from test_kernel_resources import READELF, kernels  # noqa: F401  (the fixture)

# kernel and template arguments, wavefronts per SIMD that its 512 registers must allow, vector registers it may spill
WAVES = [("gemm_fp8_kernelILi64ELi64E", 4, 0), ("gemm_fp8_kernelILi128ELi128E", 2, 0), ("gemm_fp8_kernelILi256ELi256ELi2ELi2ELi[23]ELi[23]ELb1E", 1, 0),
         ("gemm_fp8_kernelILi256ELi256ELi2ELi2ELi[23]ELi[23]ELb0E", 1, 40), ("gemm_fp8_rows_kernel", 2, 0), ("gemm_fp8_sum_kernel", 8, 0),
         ("quant_rows_kernel", 8, 0), ("quant_tile_kernelIDF16b", 8, 0), ("quant_tile_kernelIf", 4, 0), ("adamw_kernel", 8, 0)]


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs llvm-readelf")
@pytest.mark.parametrize("name,waves,spills", WAVES, ids=lambda v: str(v))
def test_wavefronts_per_simd(kernels, name, waves, spills):  # noqa: F811
    found = {k: v for k, v in kernels.items() if re.search(name, k)}
    assert found
    for k, (regs, spilled) in found.items():
        assert 512 // (-(-regs // 8) * 8) >= waves and spilled <= spills, (k, regs, spilled)


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs llvm-readelf")
def test_every_kernel_of_the_operators_is_listed(kernels):  # noqa: F811
    mine = [k for k in kernels if re.search("gemm_fp8|quant_(rows|tile)|adamw", k)]
    assert len(mine) > 50 and not [k for k in mine if not any(re.search(n, k) for n, _, _ in WAVES)]
