"""GPU: the AdamW step with every type of gradient, of copy and of state, bit for bit against its definition."""
import pytest
import torch

import paper_2312_08583_amd as P
from test_gpu_adamw import _check, _plan, _snapshot, _tensors

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
@pytest.mark.parametrize("copy", [F16, BF16, None], ids=["fp16", "bf16", "none"])
@pytest.mark.parametrize("grad", [F32, F16, BF16], ids=["fp32", "fp16", "bf16"])
def test_bit_for_bit(grad, copy, eight):
    T = _tensors((4099, 256, 1, 1000), eight, grad, copy, 47)
    plan, step = _plan(T, eight, copy), torch.tensor([9], dtype=torch.int32, device="cuda")
    scale = torch.tensor([0.25], device="cuda")
    for turn in range(2):
        start = _snapshot(T, eight)
        P.fp6_adamw(plan, step, 2e-3, 0.85, 0.98, 1e-7, 0.05, grad_scale=scale, seed=17)
        torch.cuda.synchronize()
        _check(T, start, eight, copy, 10 + turn, (2e-3, 0.85, 0.98, 1e-7, 0.05, 0.25), 17)
