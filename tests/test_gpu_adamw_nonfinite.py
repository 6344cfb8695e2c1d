"""GPU: what is not finite in a gradient, or overflows in it, stays in its element, in the calls that follow as well: the others of its block of 256 share a
scale with it, and keep the bits that they have where the element's gradient is zero."""
import pytest
import torch

import paper_2312_08583_amd as P
from adapters_ref import normal

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
N = 900                                     # three whole blocks and a short one
BAD = {5: float("inf"), 6: float("-inf"), 300: float("nan"), 600: 1e25, 899: float("inf")}          # (the square of 1e25 is above what fp32 holds)


def _run(eight, at, value, steps, grad=torch.float32):
    """Parameters and states after `steps` calls, the first one with `value` in the elements `at` of the gradient; and each call's parameters."""
    p, g = normal((N,), 1, sigma=0.02), normal((N,), 2, grad, 1e-2)
    if eight:
        states = [torch.zeros(N, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)]
        scales = [torch.zeros(-(-N // 256), dtype=torch.uint8, device="cuda") for _ in range(2)]
    else:
        states, scales = [torch.zeros(N, device="cuda") for _ in range(2)], [None, None]
    plan = P.fp6_adamw_plan([p], [g], [states[0]], [states[1]], *[[s] if eight else None for s in scales])
    step, seen = torch.zeros(1, dtype=torch.int32, device="cuda"), []
    for k in range(steps):
        g.copy_(normal((N,), 10 + k, grad, 1e-2))
        if k == 0:
            for i, v in zip(at, value):
                g[i] = v
        P.fp6_adamw(plan, step, 1e-3, 0.9, 0.999, 1e-8, 0.01, seed=7)
        seen.append(p.clone())
    bits = [s.view(torch.uint8) if eight else s for s in states]
    return seen, bits, scales


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
@pytest.mark.parametrize("at", [(5,), (5, 6, 300, 899)], ids=["one", "several"])
def test_neighbours_keep_their_bits_call_after_call(at, eight):
    seen, states, scales = _run(eight, at, [BAD[i] for i in at], 5)
    clean, want, want_scales = _run(eight, at, [0.0] * len(at), 5)
    rest = torch.ones(N, dtype=torch.bool, device="cuda")
    rest[list(at)] = False
    for got in seen:
        assert torch.isfinite(got[rest]).all()
    # (no block's largest number is one of those elements in the clean run: the scales are equal)
    for s, w in zip(scales, want_scales):
        assert s is None or torch.equal(s, w)
    for got, ref in list(zip(seen, clean)) + list(zip(states, want)):
        assert torch.equal(got[rest], ref[rest])


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
def test_a_square_that_overflows_leaves_the_others_second_moment_alone(grad):
    seen, states, scales = _run(True, (600,), [BAD[600]], 5, grad)
    clean, want, want_scales = _run(True, (600,), [0.0], 5, grad)
    rest = torch.ones(N, dtype=torch.bool, device="cuda")
    rest[600] = False
    assert torch.equal(scales[1], want_scales[1]) and torch.equal(states[1][rest], want[1][rest])
    # (its first moment is a number, 1e24, and the block's scale follows it: the others of the block round to zero beside it, and stay finite)
    for got in seen:
        assert torch.isfinite(got[rest]).all()
    other = torch.arange(N, device="cuda") // 256 != 600 // 256
    for got, ref in zip(seen, clean):
        assert torch.equal(got[other], ref[other])


def test_a_block_of_infinities_is_all_that_is_lost():
    at = tuple(range(256, 512))
    seen, states, scales = _run(True, at, [float("inf")] * 256, 4)
    clean, want, want_scales = _run(True, at, [0.0] * 256, 4)
    rest = torch.ones(N, dtype=torch.bool, device="cuda")
    rest[256:512] = False
    for got, ref in list(zip(seen, clean)) + list(zip(states, want)):
        assert torch.equal(got[rest], ref[rest])
    assert torch.isnan(seen[-1][256:512]).all()
