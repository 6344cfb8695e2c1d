"""GPU: the operators together, as a program uses them: a frozen layer with adapters beside it runs forward, its gradients go through the
frozen weight and into the adapters, the optimiser updates them, and the next forward pass serves the updated ones."""
import pytest
import torch

import paper_2312_08583_amd as P
from paper_2312_08583_amd import inputs
from adapters_ref import STEP, normal

pytestmark = pytest.mark.gpu


class Layer:
    """What a program keeps of one frozen layer with adapters: planes, turned planes, fp32 masters, 16-bit adapters, gradients."""

    def __init__(self, N, K, L, rank, dtype, seed):
        self.N, self.K, self.bf16 = N, K, dtype == torch.bfloat16
        self.format = P.FP6_FORMAT_E3M2_V2_BF16 if self.bf16 else P.FP6_FORMAT_E3M2
        W = inputs.weight(N, K, seed=seed, sigma=0.02, outlier_frac=0.001, device="cuda")
        self.planes = (P.fp6_quantize_pack_v2 if self.bf16 else P.fp6_quantize_pack)(W)
        self.turned = P.fp6_transpose_pack(*self.planes, N, K, format=self.format)
        self.W = (P.fp6_dequantize_v2 if self.bf16 else P.fp6_dequantize)(*self.planes, N, K)
        self.master = [normal((L, rank, K), seed + 1, sigma=K ** -0.5), normal((L, N, rank), seed + 2, sigma=0.02)]
        self.A, self.B = (m.to(dtype) for m in self.master)
        self.grads = [torch.zeros_like(m) for m in self.master]

    def forward(self, X, index, scaling):
        linear = P.fp6_linear_v2_bf16 if self.bf16 else P.fp6_linear
        Y = linear(X, *self.planes, self.N, self.K)
        hidden = torch.empty((X.shape[0], self.A.shape[1]), device="cuda")
        return P.fp6_lora(X, self.A, self.B, Y, index, scaling, hidden=hidden), hidden

    def backward(self, dY, X, hidden, index, scaling, accumulate=False):
        dX = P.fp6_linear_grad(dY, *self.turned, self.N, self.K, format=self.format)
        return P.fp6_lora_backward(dY, X, hidden, self.A, self.B, dX, index, scaling, dA=self.grads[0], dB=self.grads[1], accumulate=accumulate)[0]


def _optimiser(layers, eight):
    masters, grads = [m for l in layers for m in l.master], [g for l in layers for g in l.grads]
    copies = [c for l in layers for c in (l.A, l.B)]
    if not eight:
        states = [[torch.zeros_like(m) for m in masters] for _ in range(2)]
        return P.fp6_adamw_plan(masters, grads, *states, copies=copies)
    states = [[torch.zeros(m.shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for m in masters] for _ in range(2)]
    scales = [[torch.zeros(-(-m.numel() // 256), dtype=torch.uint8, device="cuda") for m in masters] for _ in range(2)]
    return P.fp6_adamw_plan(masters, grads, *states, *scales, copies)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["fp16", "bf16"])
def test_two_layers_gradients_against_autograd(dtype):
    """Gradients through two layers in turn, against autograd of the same function in 64 bits with the dequantized weight.  Each of the two
    layers rounds its result, its weight (16 bits here, exact numbers times a scale there), dY and dX to half a step at most: ten roundings
    on the way to the innermost gradient, whose errors add up in the mean square to sqrt(10) STEP at most; asserted: 4 STEP."""
    M, L, r = 96, 2, 16
    one, two = Layer(256, 192, L, r, dtype, 10), Layer(128, 256, L, r, dtype, 20)
    index = torch.randint(0, L, (M,), device="cuda", dtype=torch.int32)
    scaling = torch.tensor([2.0, 0.5], device="cuda")
    X, dY = normal((M, 192), 30, dtype), normal((M, 128), 31, dtype, 1e-1)
    H, h1 = one.forward(X, index, scaling)
    out, h2 = two.forward(H, index, scaling)
    dH = two.backward(dY, H, h2, index, scaling)
    dX = one.backward(dH, X, h1, index, scaling)

    ref = [t.detach().cpu().double().requires_grad_() for t in (X, one.A, one.B, two.A, two.B)]

    def layer(x, W, a, b):
        y = x @ W.cpu().double().T
        rows = []
        for m in range(M):
            i = int(index[m])
            rows.append(y[m] + float(scaling[i]) * (b[i] @ (a[i] @ x[m])))
        return torch.stack(rows)

    y = layer(layer(ref[0], one.W, ref[1], ref[2]), two.W, ref[3], ref[4])
    (y * dY.cpu().double()).sum().backward()
    rms = lambda a, b: float((a.cpu().double() - b).norm() / b.norm())  # noqa: E731
    assert rms(out, y.detach()) <= 4 * STEP[dtype]
    for got, want, what in zip([dX, *one.grads, *two.grads], ref, ("X", "A1", "B1", "A2", "B2")):
        assert rms(got, want.grad) <= 4 * STEP[dtype], (what, rms(got, want.grad))


@pytest.mark.parametrize("eight", [False, True], ids=["32", "8"])
def test_a_training_step_in_a_graph_equals_its_eager_run(eight):
    """Forward, two accumulated gradients, update, captured once and replayed: the masters, the adapters that the next pass reads and the results
    are the eager run's, bit for bit."""
    M, L, r, N, K = 40, 3, 8, 128, 192
    runs = []
    for captured in (False, True):
        layer = Layer(N, K, L, r, torch.float16, 50)
        plan, step = _optimiser([layer], eight), torch.zeros(1, dtype=torch.int32, device="cuda")
        index, scaling = torch.empty(M, dtype=torch.int32, device="cuda"), torch.ones(L, device="cuda")
        X, dY = torch.empty((M, K), dtype=torch.float16, device="cuda"), torch.empty((M, N), dtype=torch.float16, device="cuda")
        keep = {}

        def one_step():
            for part in range(2):
                keep["out"], hidden = layer.forward(X, index, scaling)
                keep["dX"] = layer.backward(dY, X, hidden, index, scaling, accumulate=part == 1)
            P.fp6_adamw(plan, step, lr=1e-2, weight_decay=0.0, seed=1)

        def fill(turn):
            X.copy_(normal((M, K), 60 + turn, torch.float16))
            dY.copy_(normal((M, N), 70 + turn, torch.float16))
            index.copy_(torch.arange(M, device="cuda", dtype=torch.int32) % (L + 1) - 1)

        results = []
        fill(0)
        one_step()
        if captured:
            torch.cuda.synchronize()
            stream = torch.cuda.Stream()
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):                  # (allocations and first-call work outside the capture)
                layer.forward(X, index, scaling)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                one_step()
        for turn in range(1, 5):
            fill(turn)
            graph.replay() if captured else one_step()
            torch.cuda.synchronize()
            results.append([t.clone() for t in (*layer.master, layer.A, layer.B, keep["out"], keep["dX"])])
        assert step.item() == 5
        runs.append(results)
    for a, b in zip(*runs):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_the_update_reaches_the_next_forward_pass():
    layer = Layer(128, 192, 1, 8, torch.float16, 80)
    plan, step = _optimiser([layer], False), torch.zeros(1, dtype=torch.int32, device="cuda")
    X, dY, scaling = normal((20, 192), 81, torch.float16), normal((20, 128), 82, torch.float16), torch.ones(1, device="cuda")
    out, hidden = layer.forward(X, None, scaling)
    layer.backward(dY, X, hidden, None, scaling)
    P.fp6_adamw(plan, step, lr=1e-2)
    after, _ = layer.forward(X, None, scaling)
    assert not torch.equal(out, after) and torch.equal(layer.A, layer.master[0].half()) and torch.equal(layer.B, layer.master[1].half())
