"""GPU: low-rank adapters beside a projection, forward, against the formula in 64 bits: every element within the bound that its own
roundings give."""
import pytest
import torch

import paper_2312_08583_amd as P
from adapters_ref import adapters, assert_within, forward, index_of, normal

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16

# M, N, K, rank, adapters, order of the rows
CASES = [
    (1, 64, 64, 8, 1, "none"),            # one tile of everything
    (1, 4096, 4096, 16, 1, "none"),       # many slices
    (1, 320, 192, 24, 3, "mixed"),
    (5, 64, 8192, 128, 2, "mixed"),
    (16, 1024, 2048, 16, 16, "mixed"),
    (16, 576, 448, 8, 300, "mixed"),      # more adapters than rows
    (17, 192, 320, 24, 3, "runs"),
    (33, 64, 128, 40, 2, "mixed"),
    (64, 256, 1024, 16, 40, "mixed"),
    (65, 256, 1024, 64, 40, "mixed"),     # beyond the rows that adapters are dealt out for
    (100, 640, 576, 96, 3, "mixed"),
    (333, 832, 704, 32, 5, "runs"),
    (1000, 128, 256, 16, 2, "mixed"),
    (2100, 256, 512, 64, 1, "none"),
    (4096, 4160, 64, 8, 7, "runs"),       # row tiles taken four at a time, columns that fill no workgroup
]


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("M,N,K,r,L,order", CASES)
def test_against_the_formula(M, N, K, r, L, order, dtype):
    X, Y = normal((M, K), 1, dtype), normal((M, N), 2, dtype)
    A, B = adapters(L, r, N, K, 3, dtype)
    index = index_of(order, M, L, 5)
    scaling = None if order == "runs" else normal((L,), 6).abs() + 0.25
    hidden = torch.full((M, r), float("nan"), device="cuda")
    before = Y.clone()
    out = P.fp6_lora(X, A, B, Y, index, scaling, hidden=hidden, out=torch.full_like(Y, float("nan")))
    want, H, err, herr = forward(X, A, B, Y, index, scaling)
    assert torch.equal(Y.view(torch.int16), before.view(torch.int16))
    assert_within(out, want, err, "out")
    assert_within(hidden, H, herr + 1e-38, "hidden")
    again = P.fp6_lora(X, A, B, Y, index, scaling)                   # into Y itself, without hidden: the same bits
    assert again is Y and torch.equal(again.view(torch.int16), out.view(torch.int16))


def test_rows_without_an_adapter_stay_bit_for_bit_and_reach_nobody():
    M, N, K, r, L = 50, 128, 256, 16, 3
    for dtype in (F16, BF16):
        X, Y = normal((M, K), 11, dtype), normal((M, N), 12, dtype)
        A, B = adapters(L, r, N, K, 13, dtype)
        index = index_of("mixed", M, L, 14)
        wild = torch.tensor([-1, L, 2 ** 31 - 1, -2 ** 31, -7], dtype=torch.int32, device="cuda")
        none = index < 0
        index[none] = wild[torch.arange(int(none.sum()), device="cuda") % 5]
        X[none] = float("nan")
        Y[none] = torch.tensor([float("nan"), -0.0], device="cuda", dtype=dtype).repeat(N // 2)
        hidden = torch.full((M, r), 7.0, device="cuda")
        out = P.fp6_lora(X, A, B, Y, index, hidden=hidden, out=torch.zeros_like(Y))
        assert torch.equal(out[none].view(torch.int16), Y[none].view(torch.int16)) and not hidden[none].any()
        rest = ~none
        want, H, err, herr = forward(X[rest], A, B, Y[rest], index[rest], None)
        assert_within(out[rest], want, err, "other rows")
        inplace = Y.clone()
        P.fp6_lora(X, A, B, inplace, index)
        assert torch.equal(inplace.view(torch.int16), out.view(torch.int16))


def test_no_row_has_an_adapter():
    X, Y = normal((20, 64), 1, F16), normal((20, 64), 2, F16)
    A, B = adapters(2, 8, 64, 64, 3, F16)
    hidden = torch.full((20, 8), 3.0, device="cuda")
    out = P.fp6_lora(X, A, B, Y, torch.full((20,), -1, dtype=torch.int32, device="cuda"), hidden=hidden, out=torch.zeros_like(Y))
    assert torch.equal(out, Y) and not hidden.any()


def test_an_infinity_or_nan_stays_in_its_row():
    for dtype in (F16, BF16):
        X, Y = normal((40, 128), 21, dtype), normal((40, 64), 22, dtype)
        A, B = adapters(2, 16, 64, 128, 23, dtype)
        index = index_of("mixed", 40, 2, 24)
        index[3], index[4], index[17] = 0, 1, 0
        clean = P.fp6_lora(X, A, B, Y, index, out=torch.empty_like(Y))
        X[3, 5], X[17, 100] = float("inf"), float("nan")
        out = P.fp6_lora(X, A, B, Y, index, out=torch.empty_like(Y))
        assert not torch.isfinite(out[3]).any() and torch.isnan(out[17]).all()
        rest = torch.ones(40, dtype=torch.bool, device="cuda")
        rest[[3, 17]] = False
        assert torch.equal(out[rest].view(torch.int16), clean[rest].view(torch.int16))


@pytest.mark.parametrize("size", [1e-7, 1e-4, 3e3])
def test_small_and_large_products_keep_their_bits(size):
    """H far below and above the range of fp16, brought back by the scaling."""
    M, N, K, r = 30, 64, 128, 16
    X, Y = normal((M, K), 31, F16, min(size, 1) ** 0.5 if size < 1 else 60.0), torch.zeros(M, N, dtype=F16, device="cuda")
    A, B = normal((1, r, K), 32, F16, size ** 0.5 if size < 1 else 600.0), normal((1, N, r), 33, F16, 0.05)
    scaling = torch.tensor([1 / size if size < 1 else 1e-5], device="cuda")
    out = P.fp6_lora(X, A, B, Y, None, scaling)
    want, H, err, _ = forward(X, A, B, torch.zeros(M, N, dtype=F16), None, scaling)
    assert size < 1 or H.abs().max() > 65504
    assert_within(out, want, err, size)


def test_group_equals_separate_calls():
    M, L = 16, 5
    for dtype in (F16, BF16):
        X, index = normal((M, 512), 41, dtype), index_of("mixed", M, L, 42)
        scaling = normal((L,), 43).abs() + 0.5
        layers = []
        for i, (N, r) in enumerate([(512, 16), (128, 16), (64, 8)]):
            layers.append((X,) + adapters(L, r, N, 512, 50 + i, dtype) + (normal((M, N), 60 + i, dtype),))
        other = normal((M, 256), 44, dtype)                          # a projection of other activations, with a higher rank
        layers.append((other,) + adapters(L, 40, 192, 256, 70, dtype) + (normal((M, 192), 71, dtype),))
        outs = P.fp6_lora_group(layers, index, scaling, outs=[torch.empty_like(l[3]) for l in layers])
        for (x, a, b, y), out in zip(layers, outs):
            want, _, err, _ = forward(x, a, b, y, index, scaling)
            assert_within(out, want, err, tuple(y.shape))
        for M2 in (1, 40, 200):
            xs = normal((M2, 512), 45, dtype)
            big = [(xs, l[1], l[2], normal((M2, l[3].shape[1]), 46, dtype)) for l in layers[:3]]
            idx = index_of("mixed", M2, L, 47)
            for (x, a, b, y), out in zip(big, P.fp6_lora_group(big, idx, scaling, outs=[torch.empty_like(l[3]) for l in big])):
                want, _, err, _ = forward(x, a, b, y, idx, scaling)
                assert_within(out, want, err, (M2, tuple(y.shape)))


def test_nothing_behind_the_rows_and_the_workspace_is_touched_and_its_contents_do_not_matter():
    for M, N, K, r, L in [(1, 64, 128, 8, 1), (19, 192, 256, 24, 3), (130, 320, 448, 16, 2)]:
        X = normal((M, K), 81, F16)
        A, B = adapters(L, r, N, K, 82, F16)
        index = index_of("mixed", M, L, 83)
        need = P.fp6_lora_workspace_bytes(M, N, K, r, L)
        results = []
        for fill in (0, 255):
            ws = torch.full((need + 512,), 0xA5, dtype=torch.uint8, device="cuda")
            ws[:need] = fill
            ws[:4259840] = 0
            Y = torch.full((M + 3, N), 5.0, dtype=F16, device="cuda")
            Y[:M] = normal((M, N), 84, F16)
            hidden = torch.full((M + 3, r), 9.0, device="cuda")
            P.fp6_lora(X, A, B, Y[:M], index, hidden=hidden[:M], workspace=ws[:need])
            assert (Y[M:] == 5).all() and (hidden[M:] == 9).all() and (ws[need:] == 0xA5).all() and not ws[:4259840].any()
            results.append(Y[:M].clone())
        assert torch.equal(results[0].view(torch.int16), results[1].view(torch.int16))


def test_captured_and_replayed_with_new_rows_adapters_and_owners():
    M, N, K, r, L = 24, 256, 512, 16, 6
    X, Y, out = normal((M, K), 91, F16), normal((M, N), 92, F16), torch.empty(M, N, dtype=F16, device="cuda")
    A, B = adapters(L, r, N, K, 93, F16)
    index, scaling = index_of("mixed", M, L, 94), torch.ones(L, device="cuda")
    ws = P.new_workspace(P.fp6_lora_workspace_bytes(M, N, K, r, L), "cuda")
    P.fp6_lora(X, A, B, Y, index, scaling, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.fp6_lora(X, A, B, Y, index, scaling, out=out, workspace=ws)
    for turn in range(4):
        X.copy_(normal((M, K), 100 + turn, F16))
        B.copy_(normal((L, N, r), 110 + turn, F16, 0.05))
        index.copy_(index_of("mixed", M, L, 120 + turn))
        graph.replay()
        torch.cuda.synchronize()
        eager = P.fp6_lora(X, A, B, Y, index, scaling, out=torch.empty_like(out))
        assert torch.equal(eager.view(torch.int16), out.view(torch.int16))
        want, _, err, _ = forward(X, A, B, Y, index, scaling)
        assert_within(out, want, err, turn)


def test_two_streams_with_workspaces_of_their_own():
    M, N, K, r, L = 200, 512, 1024, 32, 3
    A, B = adapters(L, r, N, K, 131, BF16)
    jobs = []
    for i in range(2):
        jobs.append((normal((M, K), 132 + i, BF16), normal((M, N), 134 + i, BF16), index_of("mixed", M, L, 136 + i),
                     P.new_workspace(P.fp6_lora_workspace_bytes(M, N, K, r, L), "cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = []
    for X, Y, index, ws, stream in jobs:
        with torch.cuda.stream(stream):
            for _ in range(3):
                out = P.fp6_lora(X, A, B, Y, index, out=torch.empty_like(Y), workspace=ws)
            outs.append(out)
    torch.cuda.synchronize()
    for (X, Y, index, _, _), out in zip(jobs, outs):
        want, _, err, _ = forward(X, A, B, Y, index, None)
        assert_within(out, want, err, "stream")


def test_refusals_of_the_binding():
    X, Y = normal((4, 64), 1, F16), normal((4, 128), 2, F16)
    A, B = adapters(2, 8, 128, 64, 3, F16)
    index, scaling = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(2, device="cuda")
    for call in [lambda: P.fp6_lora(X.float(), A, B, Y), lambda: P.fp6_lora(X, A.bfloat16(), B, Y), lambda: P.fp6_lora(X, A, B, Y[:3]),
                 lambda: P.fp6_lora(X[:, :32], A, B, Y), lambda: P.fp6_lora(X, A, B.transpose(1, 2), Y),
                 lambda: P.fp6_lora(X, A[:, :4], B[:, :, :4], Y), lambda: P.fp6_lora(X, A, B, Y, index.long()),
                 lambda: P.fp6_lora(X, A, B, Y, index[:3]), lambda: P.fp6_lora(X, A, B, Y, index, scaling[:1]),
                 lambda: P.fp6_lora(X, A, B, Y, hidden=torch.zeros(4, 16, device="cuda")), lambda: P.fp6_lora(X, A[0], B[0], Y),
                 lambda: P.fp6_lora(X, A, B, Y, out=X), lambda: P.fp6_lora(X, A, B, Y.cpu()),
                 lambda: P.fp6_lora(X, A, B, Y, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda")),
                 lambda: P.fp6_lora(torch.cat([X, X])[::2], A, B, Y),
                 lambda: P.fp6_lora_group([(X, A, B, Y), (X, A, B, Y)]), lambda: P.fp6_lora_group([(X, A, B, Y)] * 5)]:
        with pytest.raises(P.Fp6Error):
            call()
