"""GPU: the gradient of a frozen layer by its input.  The turned planes hold the same codes bit for bit; the product is held to the
formula in 64 bits, every element within the bound that its roundings give."""
import pytest
import torch

import paper_2312_08583_amd as P
from paper_2312_08583_amd import inputs
from adapters_ref import STEP, TINY, assert_within, depth, normal

pytestmark = pytest.mark.gpu

FORMATS = {"fp6": (P.FP6_FORMAT_E3M2, P.fp6_quantize_pack, P.fp6_unpack_codes), "fp5": (P.FP6_FORMAT_E3M1, P.fp5_quantize_pack, P.fp5_unpack_codes),
           "v2": (P.FP6_FORMAT_E3M2_V2, P.fp6_quantize_pack_v2, P.fp6_unpack_codes_v2),
           "bf16": (P.FP6_FORMAT_E3M2_V2_BF16, P.fp6_quantize_pack_v2, P.fp6_unpack_codes_v2)}


def _unpack(fmt, hi, lo, N, K):
    return FORMATS[fmt][2](hi, lo, N, K)


def _values(codes, fmt):
    """Codes to the numbers they stand for, from the definition (three exponent bits, bias 3)."""
    bits = 1 if fmt == "fp5" else 2
    c = codes.cpu().to(torch.int64)
    e, m = (c >> bits) & 7, (c & ((1 << bits) - 1)).double() / (1 << bits)
    v = torch.where(e > 0, (1 + m) * 2.0 ** (e - 3).double(), m * 0.25)
    return torch.where((c >> (3 + bits)) & 1 == 1, -v, v)


def _layer(fmt, N, K, seed):
    W = inputs.weight(N, K, seed=seed, sigma=0.02, outlier_frac=0.001, device="cuda")
    W[N // 2] = 0                                                      # a row of zeros: scale 0
    W[3, 5] = -0.0
    hi, lo, scales = FORMATS[fmt][1](W)
    return hi, lo, scales, _values(_unpack(fmt, hi, lo, N, K), fmt)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("N,K", [(64, 64), (64, 320), (192, 128), (640, 1024)])
def test_turned_planes_hold_the_same_codes(fmt, N, K):
    W = normal((N, K), 5, torch.float16, 0.02)
    hi, lo, scales = FORMATS[fmt][1](W)
    hi.random_(0, 256)                                                 # every code, zeros of both signs among them
    lo.random_(0, 256)
    codes = _unpack(fmt, hi, lo, N, K)
    hi_t, lo_t, scales_t, ratio = P.fp6_transpose_pack(hi, lo, scales, N, K, format=FORMATS[fmt][0])
    assert torch.equal(_unpack(fmt, hi_t, lo_t, K, N), codes.T)
    power = scales_t[0].item()
    assert (scales_t == power).all() and torch.log2(scales_t[0].double()).frac() == 0
    assert power >= scales.max().item() and power < 2 * scales.max().item()
    assert torch.equal(ratio.double() * power, scales.double())


def test_scales_at_the_ends():
    hi, lo = torch.zeros(64 * 32, dtype=torch.uint8, device="cuda"), torch.zeros(64 * 16, dtype=torch.uint8, device="cuda")
    for top, power in [(0.0, 1.0), (2.0 ** -24, 2.0 ** -24), (3 * 2.0 ** -24, 2.0 ** -22), (1.0, 1.0), (1.001, 2.0), (2340.0, 4096.0), (60000.0, 32768.0)]:
        scales = torch.zeros(64, dtype=torch.float16, device="cuda")
        scales[17] = top
        _, _, scales_t, ratio = P.fp6_transpose_pack(hi, lo, scales, 64, 64)
        assert scales_t.unique().tolist() == [power], top
        assert ratio[17].item() * power == scales[17].item() and not ratio[:17].any()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K", [(1, 64, 64), (1, 1024, 2048), (7, 192, 320), (16, 2048, 512), (33, 448, 1024), (130, 1024, 640),
                                   (515, 704, 512), (70, 8192, 128)])
def test_against_the_formula(fmt, M, N, K):
    form, dtype = FORMATS[fmt][0], torch.bfloat16 if fmt == "bf16" else torch.float16
    hi, lo, scales, values = _layer(fmt, N, K, 11)
    dY = normal((M, N), 12, dtype, 2e-2)
    planes = P.fp6_transpose_pack(hi, lo, scales, N, K, format=form)
    dX = P.fp6_linear_grad(dY, *planes, N, K, format=form)
    W = scales.cpu().double()[:, None] * values
    g = dY.cpu().double()
    want, size = g @ W, g.abs() @ W.abs()
    # dY * ratio rounded (relative, or in the smallest numbers of the type), the sum, the result
    err = (STEP[dtype] + depth(N)) * size + TINY[dtype] * float(planes[2][0]) * values.abs().sum(0)
    assert_within(dX, want, err * (1 + 2 * STEP[dtype]) + want.abs() * STEP[dtype] + TINY[dtype], fmt)
    # and in the mean square: two roundings of half a step at most, the first independent from product to product
    rms = ((dX.cpu().double() - want) ** 2).mean().sqrt() / (want ** 2).mean().sqrt()
    assert M * K < 1000 or rms <= 1.5 * STEP[dtype]


@pytest.mark.parametrize("fmt", ["fp6", "bf16"])
def test_workspace_is_shared_with_the_layer_and_left_as_the_contract_says(fmt):
    form, dtype = FORMATS[fmt][0], torch.bfloat16 if fmt == "bf16" else torch.float16
    N, K = 512, 2048
    hi, lo, scales, _ = _layer(fmt, N, K, 21)
    planes = P.fp6_transpose_pack(hi, lo, scales, N, K, format=form)
    linear = P.fp6_linear_v2_bf16 if fmt == "bf16" else P.fp6_linear
    forward_need = P.fp6_linear_v2_workspace_bytes if fmt == "bf16" else P.fp6_linear_workspace_bytes
    need = max(max(P.fp6_linear_grad_workspace_bytes(M, N, K, format=form), forward_need(M, N, K)) for M in (1, 20, 300))
    ws = torch.full((need + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    ws[:4259840] = 0
    for M in (300, 1, 20, 300):
        dY, X = normal((M, N), 22 + M, dtype, 1e-2), normal((M, K), 23 + M, dtype)
        out = torch.full((M + 1, K), 3.0, dtype=dtype, device="cuda")
        P.fp6_linear_grad(dY, *planes, N, K, format=form, out=out[:M], workspace=ws[:need])
        y = linear(X, hi, lo, scales, N, K, workspace=ws[:need])
        assert not ws[:4259840].any() and (ws[need:] == 0xA5).all() and (out[M:] == 3).all()
        assert torch.equal(out[:M].view(torch.int16), P.fp6_linear_grad(dY, *planes, N, K, format=form).view(torch.int16))
        assert torch.equal(y.view(torch.int16), linear(X, hi, lo, scales, N, K).view(torch.int16))


def test_captured_and_replayed():
    N, K, M = 1024, 512, 48
    hi, lo, scales, _ = _layer("fp6", N, K, 31)
    planes = P.fp6_transpose_pack(hi, lo, scales, N, K)
    dY, out = normal((M, N), 32, torch.float16), torch.empty((M, K), dtype=torch.float16, device="cuda")
    ws = P.new_workspace(P.fp6_linear_grad_workspace_bytes(M, N, K), "cuda")
    P.fp6_linear_grad(dY, *planes, N, K, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.fp6_linear_grad(dY, *planes, N, K, out=out, workspace=ws)
    for turn in range(4):
        dY.copy_(normal((M, N), 40 + turn, torch.float16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, P.fp6_linear_grad(dY, *planes, N, K))


def test_an_infinity_stays_in_its_row():
    N, K = 128, 192
    hi, lo, scales, _ = _layer("fp6", N, K, 51)
    planes = P.fp6_transpose_pack(hi, lo, scales, N, K)
    dY = normal((20, N), 52, torch.float16)
    clean = P.fp6_linear_grad(dY, *planes, N, K)
    dY[4, 9], dY[11, 100] = float("inf"), float("nan")
    dX = P.fp6_linear_grad(dY, *planes, N, K)
    rest = [i for i in range(20) if i not in (4, 11)]
    assert torch.equal(dX[rest], clean[rest]) and not torch.isfinite(dX[4]).any() and torch.isnan(dX[11]).all()


def test_refusals_of_the_binding():
    hi, lo, scales, _ = _layer("fp6", 128, 64, 41)
    planes = P.fp6_transpose_pack(hi, lo, scales, 128, 64)
    dY = normal((4, 128), 42, torch.float16)
    for call in [lambda: P.fp6_transpose_pack(hi, lo, scales, 64, 64), lambda: P.fp6_transpose_pack(hi, lo, scales.float(), 128, 64),
                 lambda: P.fp6_transpose_pack(hi, lo, scales, 128, 64, format=2),
                 lambda: P.fp6_linear_grad(dY.bfloat16(), *planes, 128, 64), lambda: P.fp6_linear_grad(dY[:, :64], *planes, 128, 64),
                 lambda: P.fp6_linear_grad(dY, *planes, 64, 128), lambda: P.fp6_linear_grad(dY, *planes, 128, 64, out=dY),
                 lambda: P.fp6_linear_grad(dY, *planes, 128, 64, format=3), lambda: P.fp6_linear_grad(dY.cpu(), *planes, 128, 64),
                 lambda: P.fp6_linear_grad(dY, *planes, 128, 64, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda"))]:
        with pytest.raises(P.Fp6Error):
            call()
