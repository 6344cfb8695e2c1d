"""Host-side guard on the generated code of the adapters' long kernels (needs hipcc, no GPU): as many of their workgroups fit a compute unit as their
plans count on, for both types and every class of ranks.  Two workgroups of four wavefronts have 256 registers each, and 80 KB of LDS."""
import re
import shutil

import pytest

from test_codegen_guard import _kernel_field

# JT of lora_outer_kernel and lora_second_kernel: ranks up to 16 JT.  Columns by 64: 2 or 4.
TWO = [r"lora_outer_kernelILi[68]ELi[12]ELi[24]ELb[01]ELb[01]E", r"lora_second_kernelILi[68]ELi[12]ELi[24]ELb[01]E",
       r"lora_outer_kernelILi[68]ELi4ELi2ELb[01]ELb0E", r"lora_second_kernelILi[68]ELi4ELi2ELb[01]E", r"lora_outer_kernelILi8ELi4ELi4ELb[01]ELb0E",
       r"lora_shrink_kernelILi[68]ELi[124]ELi4ELb[01]E", r"lora_expand_kernelILi[68]ELi[12]ELb[01]ELb0ELb0ELi2E"]
# counted as one, or as two against what fits, with both sides measured where the plan is made
ONE = [r"lora_outer_kernelILi[68]ELi8E", r"lora_second_kernelILi[68]ELi8E", r"lora_outer_kernelILi6ELi4ELi4E", r"lora_second_kernelILi[68]ELi4ELi4ELb0E"]


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_as_many_workgroups_fit_as_the_plans_count_on():
    regs, lds = _kernel_field("fp6_lora.hip", "vgpr_count"), _kernel_field("fp6_lora.hip", "group_segment_fixed_size")
    for pattern in TWO:
        found = {k: (v, lds[k]) for k, v in regs.items() if re.search(pattern, k)}
        assert len(found) >= 2 and all(v <= 256 and size <= 80 << 10 for v, size in found.values()), (pattern, found)
    for pattern in ONE:
        assert len([k for k in regs if re.search(pattern, k)]) >= 2, pattern
    # no outer product, and no second step, that neither list knows
    assert not [k for k in regs if re.search("lora_(outer|second)_kernel", k) and not any(re.search(p, k) for p in TWO + ONE)]
