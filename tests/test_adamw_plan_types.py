"""Host: the plan of an AdamW step holds what its addresses were worked out with, the types of gradients and copies among it."""
import ctypes

import pytest

from paper_2312_08583_amd import binding as B
from test_adapters_host import _tensor

HEADER = 128                              # the first line of a plan, before the counters of its workgroups


def _line(bits, grad, copy):
    t, _ = _tensor(0x7000_0000_0000, 4096, bits)
    arr = (B.AdamWTensor * 1)(t)
    host = (ctypes.c_uint8 * int(B.lib().fp6_adamw_plan_bytes(arr, 1)))()
    items = ctypes.c_int64()
    assert B.lib().fp6_adamw_plan(arr, 1, bits, grad, copy, ctypes.addressof(host), len(host), ctypes.byref(items)) == 0
    return bytes(host[:HEADER])


@pytest.mark.parametrize("bits", [8, 32])
def test_the_header_tells_plans_of_other_types_apart(bits):
    kinds = [(grad, copy) for grad in (B.FP6_F16, B.FP6_BF16, B.FP6_F32) for copy in (B.FP6_F16, B.FP6_BF16, B.FP6_NO_COPY)]
    lines = {_line(bits, *kind) for kind in kinds}
    assert len(lines) == len(kinds) and _line(bits, *kinds[0]) in lines
    assert not lines & {_line(40 - bits, *kind) for kind in kinds}
