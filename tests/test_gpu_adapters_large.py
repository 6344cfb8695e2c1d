"""GPU: the operators around the frozen layer where offsets pass 32 bits, and with more rows than 16 bits count.  Parts of the results are
compared: the ends, which a wrapped offset would miss or overwrite."""
import numpy as np
import pytest
import torch

import paper_2312_08583_amd as P
from adapters_ref import adapters, assert_within, backward, forward, index_of, normal
from test_gpu_adamw import _decode, _emulate

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def test_adapters_beyond_two_to_the_thirty_first_element():
    L, r, K, N, M = 520, 64, 65536, 64, 6                              # A: 2.2e9 elements
    A = torch.zeros((L, r, K), dtype=F16, device="cuda")
    B = normal((L, N, r), 1, F16, 0.05)
    owners = [0, 511, 519, 512, 519, -1]
    for a in set(owners) - {-1}:
        A[a] = normal((r, K), 10 + a, F16, K ** -0.5)
    X, Y = normal((M, K), 2, F16), normal((M, N), 3, F16)
    index = torch.tensor(owners, dtype=torch.int32, device="cuda")
    hidden = torch.empty((M, r), device="cuda")
    out = P.fp6_lora(X, A, B, Y, index, hidden=hidden, out=torch.empty_like(Y))
    small = torch.tensor([0, 1, 2, 3, 2, -1], dtype=torch.int32)
    pick = [0, 511, 519, 512]
    want, H, err, herr = forward(X, A[pick], B[pick], Y, small, None)
    assert_within(out, want, err, "out")
    assert_within(hidden, H, herr + 1e-38, "hidden")
    dY, dX = normal((M, N), 4, F16), normal((M, K), 5, F16)
    got, dA, dB = P.fp6_lora_backward(dY, X, hidden, A, B, dX, index, out=torch.empty_like(dX))
    want, err = backward(dY, X, hidden, A[pick], B[pick], dX, small, None)
    for g, w, e, what in zip((got, dA[pick], dB[pick]), want, err, ("dX", "dA", "dB")):
        assert_within(g, w, e + 1e-38, what)
    assert not dA[[1, 255, 510, 518]].any()


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
def test_activations_beyond_two_to_the_thirty_first_element(dtype):
    M, N, K, r, L = 33000, 66048, 64, 8, 2                             # Y: 2.2e9 elements
    X, A, B = normal((M, K), 1, dtype), *adapters(L, r, N, K, 2, dtype)
    index = index_of("runs", M, L, 3)
    Y = torch.empty((M, N), dtype=dtype, device="cuda")
    for at in range(0, M, 3300):
        Y[at:at + 3300] = normal((min(3300, M - at), N), 4 + at, dtype)
    before, hidden = Y[-40:].clone(), torch.empty((M, r), device="cuda")
    middle = Y[16000:16010].clone()
    P.fp6_lora(X, A, B, Y, index, hidden=hidden)
    for rows, y in ((slice(M - 40, M), before), (slice(16000, 16010), middle)):
        want, H, err, herr = forward(X[rows], A, B, y, index[rows], None)
        assert_within(Y[rows], want, err, "out")
        assert_within(hidden[rows], H, herr + 1e-38, "hidden")
    # the gradients with Y as dY: rows of dX, and columns of dB, at the end
    dX, dA, dB = P.fp6_lora_backward(Y, X, hidden, A, B, torch.zeros_like(X), index)
    want, err = backward(Y[-40:], X[-40:], hidden[-40:], A, B, torch.zeros(40, K, dtype=dtype), index[-40:], None)
    assert_within(dX[-40:], want[0], err[0], "dX")
    cols = slice(N - 64, N)
    want, err = backward(Y[:, cols], X, hidden, A, B[:, cols], torch.zeros(M, K, dtype=dtype), index, None)
    assert_within(dB[:, cols], want[2], err[2], "dB")


def test_many_rows():
    M, N, K, r, L = 70001, 64, 128, 16, 3
    X, Y = normal((M, K), 1, BF16), normal((M, N), 2, BF16)
    A, B = adapters(L, r, N, K, 3, BF16)
    index, hidden = index_of("mixed", M, L, 4), torch.empty((M, r), device="cuda")
    out = P.fp6_lora(X, A, B, Y, index, hidden=hidden, out=torch.empty_like(Y))
    want, H, err, herr = forward(X, A, B, Y, index, None)
    assert_within(out, want, err, "out")
    assert_within(hidden, H, herr + 1e-38, "hidden")
    dY, dX = normal((M, N), 5, BF16, 1e-2), normal((M, K), 6, BF16, 1e-2)
    got = P.fp6_lora_backward(dY, X, hidden, A, B, dX, index, out=torch.empty_like(dX))
    want, err = backward(dY, X, hidden, A, B, dX, index, None)
    for g, w, e, what in zip(got, want, err, ("dX", "dA", "dB")):
        assert_within(g, w, e + (1e-38 if what != "dX" else 0), what)


def test_gradient_of_a_layer_beyond_two_to_the_thirty_first_element():
    M, N, K = 17000, 128, 131072                                       # dX: 2.2e9 elements
    hi, lo, scales = P.fp6_quantize_pack(normal((N, K), 1, F16, 0.02))
    planes = P.fp6_transpose_pack(hi, lo, scales, N, K)
    dY = normal((M, N), 2, F16)
    dX = P.fp6_linear_grad(dY, *planes, N, K)
    W = P.fp6_dequantize(hi, lo, scales, N, K).cpu().double()          # (rounded to 2^-11 of each weight; dY * ratio to as much; then the result)
    for rows in (slice(0, 4), slice(M - 4, M)):
        g = dY[rows].cpu().double()
        bound = 2.5 * 2.0 ** -11 * (g.abs() @ W.abs()) + 2.0 ** -11 * (g @ W).abs() + 2.0 ** -24
        assert ((dX[rows].cpu().double() - g @ W).abs() <= bound).all()


def test_an_update_beyond_two_to_the_thirty_first_element():
    n = 2 ** 31 + 4096 + 77
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=F16, device="cuda")
    states = [torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.zeros(-(-n // 256), dtype=torch.uint8, device="cuda") for _ in range(2)]
    tail = 4096 + 77
    for at in (0, n - tail):
        p[at:at + tail] = normal((tail,), 1 + at % 7)
        g[at:at + tail] = normal((tail,), 2 + at % 7).half()
    plan, step = P.fp6_adamw_plan([p], [g], [states[0]], [states[1]], [scales[0]], [scales[1]]), torch.zeros(1, dtype=torch.int32, device="cuda")
    start = {at: (p[at:at + tail].cpu().numpy(), g[at:at + tail].float().cpu().numpy()) for at in (0, n - tail)}
    P.fp6_adamw(plan, step, 1e-3, 0.9, 0.999, 1e-8, 0.01, seed=4)
    for at, (p0, g0) in start.items():
        zero = (np.zeros(tail, np.uint8), np.zeros(-(-tail // 256), np.uint8))
        # (a block of 256 begins at the tail: 2^31 is a multiple)
        want, m, u = _emulate(p0, g0, zero, zero, 1, 1e-3, 0.9, 0.999, 1e-8, 0.01, 1.0, True, at, 4)
        assert np.array_equal(p[at:at + tail].cpu().numpy(), want)
        for s, sc, (codes, sb) in zip(states, scales, (m, u)):
            got, gs = s[at:at + tail].view(torch.uint8).cpu().numpy(), sc[at // 256:at // 256 + -(-tail // 256)].cpu().numpy()
            assert np.array_equal(gs, sb) and np.array_equal(got, codes)
            assert np.array_equal(_decode(got, gs, tail), _decode(codes, sb, tail))
    assert not p[tail:n - tail:1 << 20].any() and step.item() == 1
