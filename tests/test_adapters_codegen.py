"""Host-side guard on the generated code of the operators around the frozen layer (needs hipcc, no GPU): their loops keep loads in flight in
registers, and a spilled register is read back between them (the shrink kernel with several ways out of its loop held its sums twice
and took 76 us instead of 36 at 2048 x 22016, rank 64)."""
import shutil

import pytest

from test_codegen_guard import _kernel_field


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
@pytest.mark.parametrize("source,kernels", [("fp6_lora.hip", "lora_"), ("fp6_adamw.hip", "adamw_kernel"), ("fp6_grad.hip", "_kernel")])
def test_kernels_do_not_spill(source, kernels):
    sizes = {k: v for k, v in _kernel_field(source, "private_segment_fixed_size").items() if kernels in k}
    assert sizes and all(v == 0 for v in sizes.values()), {k: v for k, v in sizes.items() if v}


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_two_workgroups_of_the_long_kernels_fit_a_compute_unit():
    """Their plans count on two workgroups of four wavefronts to a unit: 256 of a SIMD's 512 registers, for ranks up to 32."""
    regs = _kernel_field("fp6_lora.hip", "vgpr_count")
    long = {k: v for k, v in regs.items() if "lora_outer_kernelILi6ELi1E" in k or "lora_second_kernelILi6ELi1E" in k or
            "lora_shrink_kernelILi6ELi1ELi4" in k or "lora_shrink_kernelILi6ELi2ELi4" in k or "lora_expand_kernelILi6ELi1ELb1ELb0ELb0" in k}
    assert len(long) >= 6 and all(v <= 256 for v in long.values()), long
