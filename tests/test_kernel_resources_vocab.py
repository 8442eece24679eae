"""Register budgets of the vocabulary operators' kernels (see test_kernel_resources.py): a row of logits stays in registers
between its statistics and its gradient, and sixteen rows of activations are in flight."""
import os
import re

import pytest

from test_kernel_resources import READELF, kernels  # noqa: F401  (the fixture)

# kernel and template arguments, wavefronts per SIMD that its 512 registers must allow, vector registers it may spill
WAVES = [("distill_rows_kernelI(DF16b|f)Li(64|128|256)ELi4E", 8, 0), ("distill_rows_kernelI(DF16b|f)Li256ELi8E", 6, 0),
         ("distill_rows_kernelI(DF16b|f)Li(256|512)ELi16E", 4, 0), ("distill_rows_kernelI(DF16b|f)Li1024ELi16ELi[0-3]ELi0ELb0E", 4, 0),
         # (four wavefronts a SIMD are its own 1024 threads: it may have 128 registers and wants some ten more)
         ("distill_rows_kernelI(DF16b|f)Li1024ELi16ELi[0-3]ELi0ELb1E", 4, 10),
         ("top_logits_kernelI(DF16b|f)Li64ELi(4|16)ELb1E", 8, 0), ("top_logits_kernelI(DF16b|f)Li(64|128)ELi8E", 8, 0),
         ("top_logits_kernelI(DF16b|f)Li(128|256)ELi16ELb1E", 7, 0), ("top_logits_kernelI(DF16b|f)Li256ELi4ELb0E", 6, 1),
         ("top_logits_kernelI(DF16b|f)Li(64|128|256)ELi16ELb0E", 4, 0), ("top_logits_kernelI(DF16b|f)Li256ELi16ELb0E", 5, 0),
         ("top_logits_kernelI(DF16b|f)Li1024ELi16ELb0E", 4, 0),
         ("embed_tile_sum_kernel", 4, 0), ("embed_join_kernel", 7, 0), ("embed_owner_sum_kernel", 6, 0), ("embed_sort_", 8, 0),
         ("embed_scaled_fwd_kernel", 8, 0)]


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs llvm-readelf")
@pytest.mark.parametrize("name,waves,spills", WAVES, ids=lambda v: str(v))
def test_wavefronts_per_simd(kernels, name, waves, spills):  # noqa: F811
    found = {k: v for k, v in kernels.items() if re.search(name, k)}
    assert found
    for k, (regs, spilled) in found.items():
        assert 512 // (-(-regs // 8) * 8) >= waves and spilled <= spills, (k, regs, spilled)


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs llvm-readelf")
def test_every_kernel_of_the_operators_is_listed(kernels):  # noqa: F811
    mine = [k for k in kernels if re.search("distill_rows|top_logits_kernel|embed_(tile|join|owner|sort|scaled)", k)]
    assert len(mine) > 100 and not [k for k in mine if not any(re.search(n, k) for n, _, _ in WAVES)]
