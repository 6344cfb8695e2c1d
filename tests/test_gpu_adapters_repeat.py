"""GPU: the same call again gives the same bits, forward and backward, with rows of many adapters in any order and one call right after another
(few rows: several workgroups share the rows, each with an adapter of its own)."""
import pytest
import torch

import paper_2312_08583_amd as P
from adapters_ref import adapters, assert_within, forward, index_of, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("M,N,K,r,L", [(16, 1024, 2048, 16, 16), (16, 1024, 4096, 16, 16), (13, 512, 2048, 8, 5), (64, 512, 8192, 32, 16),
                                       (200, 512, 4096, 16, 9), (300, 512, 4096, 64, 9), (700, 512, 4096, 16, 9)])
def test_the_same_call_gives_the_same_bits(M, N, K, r, L, dtype):
    X, Y, dX = normal((M, K), 1, dtype), normal((M, N), 2, dtype), normal((M, K), 7, dtype)
    A, B = adapters(L, r, N, K, 3, dtype)
    index = index_of("mixed", M, L, 4)

    def step():
        hidden = torch.empty((M, r), device="cuda")
        out = P.fp6_lora(X, A, B, Y, index, hidden=hidden, out=torch.empty_like(Y))
        return [hidden, out, *P.fp6_lora_backward(out, X, hidden, A, B, dX, index, out=torch.empty_like(dX))]

    first = step()
    want, H, err, herr = forward(X, A, B, Y, index, None)
    assert_within(first[1], want, err, "out")
    assert_within(first[0], H, herr + 1e-38, "hidden")
    for _ in range(50):
        for a, b in zip(first, step()):
            assert torch.equal(a, b)
