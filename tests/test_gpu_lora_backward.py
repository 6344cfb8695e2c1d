"""GPU: the gradients of low-rank adapters, against the formula in 64 bits and against differences."""
import pytest
import torch

import paper_2312_08583_amd as P
from adapters_ref import adapters, assert_within, backward, forward, index_of, normal

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16

CASES = [
    (1, 64, 64, 8, 1, "none"),
    (3, 192, 64, 24, 2, "mixed"),
    (40, 1024, 1024, 8, 1, "none"),
    (64, 64, 320, 16, 3, "mixed"),
    (65, 320, 128, 128, 1, "none"),
    (100, 704, 576, 32, 2, "runs"),
    (200, 128, 192, 72, 5, "mixed"),
    (777, 256, 512, 64, 3, "runs"),
    (2048, 512, 128, 16, 1, "none"),      # ranges of rows for workgroups of their own
    (3000, 192, 320, 40, 40, "mixed"),
    (1500, 4160, 4224, 16, 2, "runs"),
]


def _inputs(M, N, K, r, L, order, dtype, seed=1):
    X, dY, dX = normal((M, K), seed, dtype), normal((M, N), seed + 1, dtype, 1e-2), normal((M, K), seed + 2, dtype, 1e-2)
    A, B = adapters(L, r, N, K, seed + 3, dtype)
    index = index_of(order, M, L, seed + 5)
    scaling = None if order == "runs" else normal((L,), seed + 6).abs() + 0.25
    hidden = torch.empty((M, r), device="cuda")
    P.fp6_lora(X, A, B, normal((M, N), seed + 7, dtype), index, scaling, hidden=hidden)
    return dY, X, hidden, A, B, dX, index, scaling


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("M,N,K,r,L,order", CASES)
def test_against_the_formula(M, N, K, r, L, order, dtype):
    args = _inputs(M, N, K, r, L, order, dtype)
    dX, index, scaling = args[5:]
    before = dX.clone()
    got = P.fp6_lora_backward(*args[:5], dX, index, scaling, out=torch.full_like(dX, float("nan")))
    want, err = backward(*args)
    assert torch.equal(before.view(torch.int16), dX.view(torch.int16))
    for g, w, e, what in zip(got, want, err, ("dX", "dA", "dB")):
        assert_within(g, w, e + (1e-38 if what != "dX" else 0), what)
    # added to, in place, without a gradient for X: the same sums
    dA, dB = normal(got[1].shape, 8, sigma=0.1), normal(got[2].shape, 9, sigma=0.1)
    a0, b0 = dA.clone(), dB.clone()
    none = P.fp6_lora_backward(*args[:5], None, index, scaling, dA=dA, dB=dB, accumulate=True)
    assert none[0] is None and none[1] is dA and none[2] is dB
    for total, start, e, w in ((dA, a0, err[1], want[1]), (dB, b0, err[2], want[2])):
        assert_within(total, start.cpu().double() + w, e + 2.0 ** -22 * (start.cpu().double().abs() + w.abs()) + 1e-38, "accumulated")
    inplace = P.fp6_lora_backward(*args[:5], dX, index, scaling)
    for g, i in zip(got, inplace):
        assert torch.equal(g.view(torch.int16), i.view(torch.int16))          # (bits; the order of the sums is fixed)


def test_rows_without_an_adapter_enter_nothing():
    for dtype in (F16, BF16):
        M, N, K, r, L = 150, 128, 192, 16, 3
        dY, X, hidden, A, B, dX, index, scaling = _inputs(M, N, K, r, L, "mixed", dtype, 20)
        index[index == 1] = -5                                                # an adapter without rows
        none = index < 0
        clean = P.fp6_lora_backward(dY, X, hidden, A, B, dX, index, scaling, out=torch.empty_like(dX))
        for t in (dY, X, hidden):
            t[none] = float("nan")
        dX[none] = float("inf")
        out, dA, dB = P.fp6_lora_backward(dY, X, hidden, A, B, dX, index, scaling, out=torch.empty_like(dX))
        assert torch.equal(dA, clean[1]) and torch.equal(dB, clean[2]) and not dA[1].any() and not dB[1].any()
        assert torch.equal(out[none].view(torch.int16), dX[none].view(torch.int16))
        assert torch.equal(out[~none].view(torch.int16), clean[0][~none].view(torch.int16))


def test_an_infinity_reaches_its_adapter_only():
    for dtype in (F16, BF16):
        M, N, K, r, L = 90, 64, 64, 8, 2
        dY, X, hidden, A, B, dX, index, scaling = _inputs(M, N, K, r, L, "mixed", dtype, 30)
        clean = P.fp6_lora_backward(dY, X, hidden, A, B, dX, index, scaling, out=torch.empty_like(dX))
        row = int((index == 0).nonzero()[0])
        dY[row, 7] = float("inf")
        out, dA, dB = P.fp6_lora_backward(dY, X, hidden, A, B, dX, index, scaling, out=torch.empty_like(dX))
        assert not torch.isfinite(dA[0]).any() and torch.equal(dA[1], clean[1][1])
        assert torch.equal(dB[1], clean[2][1]) and not torch.isfinite(dB[0, 7]).any()
        keep = torch.arange(N, device="cuda") != 7
        assert torch.equal(dB[0][keep], clean[2][0][keep])
        rest = torch.arange(M, device="cuda") != row
        assert torch.equal(out[rest].view(torch.int16), clean[0][rest].view(torch.int16)) and not torch.isfinite(out[row]).any()


@pytest.mark.parametrize("size", [1e-6, 1e-3, 1e3])
def test_gradients_far_from_one(size):
    """Sizes that fp16 cannot hold a dH of: 1e-6 as under no loss scale, and the other way."""
    M, N, K, r, L, dtype = 260, 128, 64, 16, 2, F16
    dY, X, hidden, A, B, dX, index, scaling = _inputs(M, N, K, r, L, "mixed", dtype, 40)
    dY, dX = normal((M, N), 41, dtype, min(size, 50.0)), torch.zeros_like(dX)
    scaling = scaling * (size / 50 if size > 50 else 1.0)
    hidden = hidden * size
    got = P.fp6_lora_backward(dY, X, hidden, A, B, dX, index, scaling)
    want, err = backward(dY, X, hidden, A, B, torch.zeros_like(X), index, scaling)
    for g, w, e, what in zip(got, want, err, ("dX", "dA", "dB")):
        assert_within(g, w, e, what)


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
def test_against_differences(dtype):
    """<dL/dp, direction> against (L(p + h d) - L(p - h d)) / 2h of L = sum(dY * out) in 64 bits.  L is linear in each of the three
    taken alone: the difference is exact but for its own rounding (1e-16 * |L| / h)."""
    M, N, K, r, L = 60, 64, 128, 16, 2
    dY, X, hidden, A, B, _, index, scaling = _inputs(M, N, K, r, L, "mixed", dtype, 50)
    hidden = forward(X, A, B, torch.zeros(M, N, dtype=dtype), index, scaling)[1].float().cuda()
    out, dA, dB = P.fp6_lora_backward(dY, X, hidden, A, B, torch.zeros_like(X), index, scaling)
    want, err = backward(dY, X, hidden, A, B, torch.zeros_like(X), index, scaling)
    Y, g = torch.zeros(M, N, dtype=dtype), dY.cpu().double()

    def loss(x, a, b):
        return float((forward(x, a, b, Y, index, scaling)[0] * g).sum())

    args = [t.cpu().double() for t in (X, A, B)]
    for which, (grad, e) in enumerate(zip((out, dA, dB), err)):
        d = normal(tuple(grad.shape), 60 + which, torch.float64, device="cpu")
        h = 2.0 ** -10
        up = [t + h * d if i == which else t for i, t in enumerate(args)]
        down = [t - h * d if i == which else t for i, t in enumerate(args)]
        difference = (loss(*up) - loss(*down)) / (2 * h)
        assert abs(float((grad.cpu().double() * d).sum()) - difference) <= float((e * d.abs()).sum()) + 1e-9 * (1 + abs(difference))


def test_nothing_behind_the_tensors_and_the_workspace_is_touched():
    for M, N, K, r, L in [(1, 64, 128, 8, 1), (131, 192, 256, 24, 3), (600, 320, 448, 16, 1)]:
        dY, X, hidden, A, B, dX, index, scaling = _inputs(M, N, K, r, L, "mixed", F16, 70)
        need = P.fp6_lora_backward_workspace_bytes(M, N, K, r, L)
        bits = []
        for fill in (0, 255):
            ws = torch.full((need + 512,), 0xA5, dtype=torch.uint8, device="cuda")
            ws[:need] = fill
            ws[:4259840] = 0
            out = torch.full((M + 2, K), 5.0, dtype=F16, device="cuda")
            dA, dB = torch.full((L + 1, r, K), 6.0, device="cuda"), torch.full((L + 1, N, r), 7.0, device="cuda")
            P.fp6_lora_backward(dY, X, hidden, A, B, dX, index, scaling, dA=dA[:L], dB=dB[:L], out=out[:M], workspace=ws[:need])
            assert (out[M:] == 5).all() and (dA[L:] == 6).all() and (dB[L:] == 7).all()
            assert (ws[need:] == 0xA5).all() and not ws[:4259840].any()
            bits.append((out.clone(), dA.clone(), dB.clone()))
        assert all(torch.equal(x, y) for x, y in zip(*bits))


def test_captured_and_replayed():
    M, N, K, r, L = 300, 256, 192, 16, 3
    dY, X, hidden, A, B, dX, index, scaling = _inputs(M, N, K, r, L, "mixed", BF16, 80)
    ws = P.new_workspace(P.fp6_lora_backward_workspace_bytes(M, N, K, r, L), "cuda")
    out, dA, dB = torch.empty_like(dX), torch.empty(L, r, K, device="cuda"), torch.empty(L, N, r, device="cuda")
    call = lambda: P.fp6_lora_backward(dY, X, hidden, A, B, dX, index, scaling, dA=dA, dB=dB, out=out, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(4):
        dY.copy_(normal((M, N), 90 + turn, BF16, 1e-2))
        index.copy_(index_of("mixed", M, L, 95 + turn))
        graph.replay()
        torch.cuda.synchronize()
        eager = P.fp6_lora_backward(dY, X, hidden, A, B, dX, index, scaling, out=torch.empty_like(dX))
        assert torch.equal(out.view(torch.int16), eager[0].view(torch.int16)) and torch.equal(dA, eager[1]) and torch.equal(dB, eager[2])


def test_refusals_of_the_binding():
    dY, X, hidden, A, B, dX, index, scaling = _inputs(8, 64, 128, 8, 2, "mixed", F16, 90)
    for call in [lambda: P.fp6_lora_backward(dY.bfloat16(), X, hidden, A, B), lambda: P.fp6_lora_backward(dY, X, hidden.half(), A, B),
                 lambda: P.fp6_lora_backward(dY, X, hidden[:, :4], A, B), lambda: P.fp6_lora_backward(dY, X, hidden, A, B, accumulate=True),
                 lambda: P.fp6_lora_backward(dY, X, hidden, A, B, out=dX), lambda: P.fp6_lora_backward(dY, X, hidden, A, B, X),
                 lambda: P.fp6_lora_backward(dY, X, hidden, A, B, dA=torch.empty(2, 8, 128, device="cuda", dtype=F16)),
                 lambda: P.fp6_lora_backward(dY, X, hidden, A, B, dX[:, ::2]), lambda: P.fp6_lora_backward(dY[:7], X, hidden, A, B)]:
        with pytest.raises(P.Fp6Error):
            call()
