"""GPU: adapters and their gradients in every kernel that ranks and numbers of rows lead to, every element against the formula in 64 bits: ranks above 64
and between 17 and 64 with few rows, with rows that pass 256 and 512, and with so many columns that more than 32 partial sums meet, or a workgroup
takes 256 of them; groups of many rows."""
import pytest
import torch

import paper_2312_08583_amd as P
from adapters_ref import adapters, assert_within, backward, forward, index_of, normal

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16

# M, N, K, rank, adapters, order
CASES = [
    (256, 192, 448, 40, 3, "mixed"),      # two launches backward, rank 33 to 64
    (100, 320, 192, 64, 1, "none"),
    (257, 192, 320, 128, 3, "mixed"),     # sixteen rows to a workgroup, the sums added up by a launch of their own
    (300, 448, 192, 72, 2, "runs"),
    (300, 320, 576, 48, 9, "mixed"),
    (512, 192, 704, 64, 4, "mixed"),
    (513, 576, 192, 128, 1, "none"),      # thirty-two rows, and ranges of rows
    (600, 320, 448, 72, 3, "mixed"),
    (1100, 192, 1088, 104, 5, "runs"),
    (300, 8256, 192, 24, 3, "mixed"),     # dB and the shrink of dY in one reading, 33 parts of dH
    (1000, 8256, 320, 32, 3, "runs"),
    (1030, 192, 8256, 24, 1, "none"),
    (777, 448, 576, 32, 7, "mixed"),
    (300, 192, 21888, 16, 3, "mixed"),    # 256 columns to a workgroup: with 128, three adapters on 171 blocks are more than 512
    (300, 192, 21888, 24, 3, "runs"),
    (300, 192, 21888, 40, 3, "mixed"),
    (300, 21888, 192, 56, 3, "mixed"),
]


def _inputs(M, N, K, r, L, order, dtype):
    X, Y = normal((M, K), 1, dtype), normal((M, N), 2, dtype)
    A, B = adapters(L, r, N, K, 3, dtype)
    index = index_of(order, M, L, 5)
    return X, Y, A, B, index, None if order == "runs" else normal((L,), 6).abs() + 0.25


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("M,N,K,r,L,order", CASES)
def test_forward(M, N, K, r, L, order, dtype):
    X, Y, A, B, index, scaling = _inputs(M, N, K, r, L, order, dtype)
    hidden = torch.full((M, r), float("nan"), device="cuda")
    out = P.fp6_lora(X, A, B, Y, index, scaling, hidden=hidden, out=torch.full_like(Y, float("nan")))
    want, H, err, herr = forward(X, A, B, Y, index, scaling)
    assert_within(out, want, err, "out")
    assert_within(hidden, H, herr + 1e-38, "hidden")
    again = P.fp6_lora(X, A, B, Y, index, scaling)
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("M,N,K,r,L,order", CASES)
def test_backward(M, N, K, r, L, order, dtype):
    X, _, A, B, index, scaling = _inputs(M, N, K, r, L, order, dtype)
    dY, dX = normal((M, N), 7, dtype, 1e-2), normal((M, K), 8, dtype, 1e-2)
    hidden = torch.empty((M, r), device="cuda")
    P.fp6_lora(X, A, B, torch.zeros(M, N, dtype=dtype, device="cuda"), index, scaling, hidden=hidden)
    args = (dY, X, hidden, A, B, dX, index, scaling)
    got = P.fp6_lora_backward(*args, out=torch.full_like(dX, float("nan")))
    want, err = backward(*args)
    for g, w, e, what in zip(got, want, err, ("dX", "dA", "dB")):
        assert_within(g, w, e + (1e-38 if what != "dX" else 0), what)
    # added to, without a gradient for X
    dA, dB = normal(got[1].shape, 9, sigma=0.1), normal(got[2].shape, 10, sigma=0.1)
    a0, b0 = dA.clone(), dB.clone()
    P.fp6_lora_backward(dY, X, hidden, A, B, None, index, scaling, dA=dA, dB=dB, accumulate=True)
    for total, start, e, w in ((dA, a0, err[1], want[1]), (dB, b0, err[2], want[2])):
        s = start.cpu().double()
        assert_within(total, s + w, e + 2.0 ** -22 * (s.abs() + w.abs()) + 1e-38, "accumulated")
    inplace = P.fp6_lora_backward(*args)
    for g, i in zip(got, inplace):
        assert torch.equal(g.view(torch.int16), i.view(torch.int16))


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("M,order", [(257, "mixed"), (300, "runs"), (600, "mixed"), (1100, "none")])
@pytest.mark.parametrize("ranks", [(16, 16, 8), (8, 40, 16, 128), (24, 8, 32)], ids=str)
def test_groups_of_many_rows(ranks, M, order, dtype):
    L = 1 if order == "none" else 4
    index, scaling = index_of(order, M, L, 21), normal((L,), 22).abs() + 0.5
    shared, other = normal((M, 576), 23, dtype), normal((M, 320), 24, dtype)
    layers = []
    for i, r in enumerate(ranks):
        X, N = (other if i == 1 else shared), (448, 64, 192, 320)[i]
        layers.append((X,) + adapters(L, r, N, X.shape[1], 30 + 2 * i, dtype) + (normal((M, N), 40 + i, dtype),))
    outs = P.fp6_lora_group(layers, index, scaling, outs=[torch.full_like(l[3], float("nan")) for l in layers])
    for (X, A, B, Y), out in zip(layers, outs):
        want, _, err, _ = forward(X, A, B, Y, index, scaling)
        assert_within(out, want, err, tuple(out.shape))
    for l, out, own in zip(layers, outs, P.fp6_lora_group(layers, index, scaling)):
        assert own is l[3] and torch.equal(own.view(torch.int16), out.view(torch.int16))
