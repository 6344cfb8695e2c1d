"""Host-only checks of the operators around the frozen layer: every refusal is made before anything is launched, workspaces are
functions of the sizes, and the optimiser's plan is what the header says."""
import ctypes

import pytest
import torch

import paper_2312_08583_amd as P
from paper_2312_08583_amd import binding as B

NULL, SHAPE, ALIGN, WORKSPACE, VARIANT, OVERLAP, VALUE = -1, -2, -3, -4, -5, -8, -9
MB = 1 << 20


def _addresses(n, spacing=64 * MB):
    """Aligned addresses that nothing lies at: every call below is refused before one is used."""
    return [0x7000_0000_0000 + i * spacing for i in range(n)]


def _lora(**change):
    a = _addresses(9)
    c = dict(type=0, X=a[0], M=4, A=a[1], B=a[2], adapters=2, rank=16, index=a[3], scaling=a[4], Y=a[5], N=128, K=192, out=a[6],
             hidden=a[7], ws=a[8], wb=8 * MB)
    c.update(change)
    return B.lib().fp6_lora(*[c[k] for k in ("type", "X", "M", "A", "B", "adapters", "rank", "index", "scaling", "Y", "N", "K", "out",
                                             "hidden", "ws", "wb")], None)


@pytest.mark.parametrize("change,status", [
    (dict(X=None), NULL), (dict(A=None), NULL), (dict(B=None), NULL), (dict(Y=None), NULL), (dict(out=None), NULL),
    (dict(M=0), SHAPE), (dict(M=-1), SHAPE), (dict(M=(1 << 24) + 1), SHAPE), (dict(N=100), SHAPE), (dict(K=0), SHAPE),
    (dict(type=2), VALUE), (dict(type=-1), VALUE), (dict(rank=0), VALUE), (dict(rank=12), VALUE), (dict(rank=136), VALUE),
    (dict(adapters=0), VALUE), (dict(adapters=65536), VALUE),
    (dict(X=0x7000_0000_0002), ALIGN), (dict(hidden=0x7000_1000_0008), ALIGN), (dict(index=0x7000_2000_0004), ALIGN),
    (dict(ws=None), WORKSPACE), (dict(wb=4 * MB), WORKSPACE), (dict(wb=0), WORKSPACE),
    (dict(out=0x7000_0000_0000), OVERLAP),                                  # out = X
    (dict(out=_addresses(9)[5] + 256), OVERLAP),                            # out beside Y, not Y
    (dict(hidden=_addresses(9)[6] + 512), OVERLAP), (dict(ws=_addresses(9)[6]), OVERLAP), (dict(out=_addresses(9)[3]), OVERLAP),
])
def test_lora_refusals(change, status):
    assert _lora(**change) == status


def _backward(**change):
    a = _addresses(12)
    c = dict(type=1, dY=a[0], X=a[1], hidden=a[2], M=4, A=a[3], B=a[4], adapters=2, rank=16, index=a[5], scaling=a[6], dX=a[7], out=a[8],
             dA=a[9], dB=a[10], acc=0, N=128, K=192, ws=a[11], wb=8 * MB)
    c.update(change)
    return B.lib().fp6_lora_backward(*[c[k] for k in ("type", "dY", "X", "hidden", "M", "A", "B", "adapters", "rank", "index", "scaling",
                                                      "dX", "out", "dA", "dB", "acc", "N", "K", "ws", "wb")], None)


@pytest.mark.parametrize("change,status", [
    (dict(dY=None), NULL), (dict(hidden=None), NULL), (dict(dA=None), NULL), (dict(dB=None), NULL), (dict(dX=None), NULL),
    (dict(out=None), NULL), (dict(M=0), SHAPE), (dict(N=65), SHAPE), (dict(type=2), VALUE), (dict(rank=4), VALUE),
    (dict(adapters=0), VALUE), (dict(dA=0x7000_3000_0004), ALIGN), (dict(ws=None), WORKSPACE), (dict(wb=1 * MB), WORKSPACE),
    (dict(dA=_addresses(12)[10]), OVERLAP), (dict(out=_addresses(12)[1]), OVERLAP), (dict(out=_addresses(12)[7] + 16), OVERLAP),
    (dict(dX=_addresses(12)[1], out=_addresses(12)[1]), OVERLAP),           # in place, but in X
    (dict(dB=_addresses(12)[0]), OVERLAP), (dict(ws=_addresses(12)[8]), OVERLAP),
])
def test_backward_refusals(change, status):
    assert _backward(**change) == status


def _grad(**change):
    a = _addresses(7)
    c = dict(format=6, dY=a[0], M=4, hi=a[1], lo=a[2], scales=a[3], ratio=a[4], N=128, K=192, dX=a[5], ws=a[6], wb=8 * MB)
    c.update(change)
    return B.lib().fp6_linear_grad(*[c[k] for k in ("format", "dY", "M", "hi", "lo", "scales", "ratio", "N", "K", "dX", "ws", "wb")], None)


@pytest.mark.parametrize("change,status", [
    (dict(dY=None), NULL), (dict(ratio=None), NULL), (dict(dX=None), NULL), (dict(format=0), VARIANT), (dict(format=9), VARIANT),
    (dict(M=0), SHAPE), (dict(N=96), SHAPE), (dict(K=-64), SHAPE), (dict(hi=0x7000_4000_0008), ALIGN), (dict(ws=None), WORKSPACE),
    (dict(wb=B.FP6_WORKSPACE_ZERO_BYTES), WORKSPACE), (dict(dX=_addresses(7)[0]), OVERLAP), (dict(dX=_addresses(7)[6] + 1024), OVERLAP),
])
def test_grad_refusals(change, status):
    assert _grad(**change) == status


def test_transpose_refusals():
    a = _addresses(7)
    f = B.lib().fp6_transpose_pack
    assert f(6, None, a[1], a[2], 64, 64, a[3], a[4], a[5], a[6], None) == NULL
    assert f(6, a[0], a[1], a[2], 64, 64, a[3], a[4], a[5], None, None) == NULL
    assert f(3, a[0], a[1], a[2], 64, 64, a[3], a[4], a[5], a[6], None) == VARIANT
    assert f(6, a[0], a[1], a[2], 64, 65, a[3], a[4], a[5], a[6], None) == SHAPE
    assert f(6, a[0] + 2, a[1], a[2], 64, 64, a[3], a[4], a[5], a[6], None) == ALIGN
    assert f(6, a[0], a[1], a[2], 64, 64, a[0], a[4], a[5], a[6], None) == OVERLAP
    assert f(6, a[0], a[1], a[2], 64, 64, a[3], a[3] + 1024, a[5], a[6], None) == OVERLAP


def test_group_refusals():
    a = _addresses(20)

    def group(problems, count=None, M=4, adapters=2, type=0, wb=32 * MB):
        arr = (B.LoraProblem * max(1, len(problems)))(*problems)
        return B.lib().fp6_lora_group(type, M, arr, len(problems) if count is None else count, adapters, None, None, a[0], wb, None)

    one = B.LoraProblem(a[1], a[2], a[3], a[4], a[5], None, 128, 192, 16)
    assert group([one], count=0) == SHAPE and group([one] * 4, count=5) == SHAPE
    assert B.lib().fp6_lora_group(0, 4, None, 1, 1, None, None, a[0], MB, None) == NULL
    assert group([one, B.LoraProblem(a[1], a[6], a[7], a[8], None, None, 64, 192, 8)]) == NULL
    assert group([one, B.LoraProblem(a[1], a[6], a[7], a[8], a[5] + 64, None, 64, 192, 8)]) == OVERLAP          # two results
    assert group([one, B.LoraProblem(a[1], a[6], a[7], a[8], a[2], None, 64, 192, 8)]) == OVERLAP               # the other's A
    assert group([one, B.LoraProblem(a[5], a[6], a[7], a[8], a[9], None, 64, 128, 8)]) == OVERLAP               # X is the other's result
    assert group([one, B.LoraProblem(a[1], a[6], a[7], a[8], a[9], None, 64, 192, 20)]) == VALUE
    assert group([one], wb=MB) == WORKSPACE


def test_workspaces_are_functions_of_the_sizes():
    zero = B.FP6_WORKSPACE_ZERO_BYTES
    for M in (1, 16, 64, 65, 1000, 70000):
        need = P.fp6_lora_workspace_bytes(M, 4096, 4096, 16, 3)
        assert need > zero and (need - zero) % 256 == 0 and (need - zero) >= 4 * M * 16
        assert P.fp6_lora_backward_workspace_bytes(M, 4096, 4096, 16, 3) > zero
        for fmt in (6, 5, 7, 8):
            assert P.fp6_linear_grad_workspace_bytes(M, 4096, 1024, format=fmt) >= zero + 2 * M * 4096
    two = P.fp6_lora_group_workspace_bytes(16, [(4096, 4096, 16), (1024, 4096, 16)], 4)
    assert two > P.fp6_lora_workspace_bytes(16, 4096, 4096, 16, 4)
    assert P.fp6_lora_workspace_bytes(0, 64, 64, 8) == 0 and P.fp6_lora_workspace_bytes(1, 64, 64, 9) == 0
    # more workgroups than a launch counts: refused before anything is launched
    assert P.fp6_lora_workspace_bytes(64, 1 << 22, 64, 8, 16) > 0 and P.fp6_lora_workspace_bytes(64, 1 << 24, 64, 8, 16) == 0
    assert P.fp6_lora_workspace_bytes(256, 1 << 24, 64, 8, 4) == 0 and P.fp6_lora_workspace_bytes(1 << 20, 1 << 18, 64, 8, 4) == 0
    assert P.fp6_lora_backward_workspace_bytes(64, 64, 16448, 8, 65535) == 0 and P.fp6_lora_backward_workspace_bytes(64, 64, 8192, 8, 65535) > 0
    assert P.fp6_lora_backward_workspace_bytes(1, 64, 65, 8) == 0 and P.fp6_linear_grad_workspace_bytes(1, 64, 64, format=1) == 0


def _tensor(at, count, bits=32, copy=True):
    s = 1 if bits == 8 else 4
    spans = [4 * count, 4 * count, s * count, s * count, -(-count // 256), -(-count // 256), 2 * count]
    p = []
    for size in spans:
        p.append(at)
        at += (size + 15) // 16 * 16
    return B.AdamWTensor(p[0], p[1], p[2], p[3], p[4] if bits == 8 else None, p[5] if bits == 8 else None, p[6] if copy else None, count), at


def _plan(tensors, bits=32, grad=2, copy=0, nbytes=None):
    arr = (B.AdamWTensor * len(tensors))(*tensors)
    need = int(B.lib().fp6_adamw_plan_bytes(arr, len(tensors)))
    host = (ctypes.c_uint8 * max(need, 64))()
    items = ctypes.c_int64(-1)
    rc = B.lib().fp6_adamw_plan(arr, len(tensors), bits, grad, copy, ctypes.addressof(host), need if nbytes is None else nbytes,
                                ctypes.byref(items))
    return rc, items.value


@pytest.mark.parametrize("bits", [8, 32])
def test_plan_counts_items_and_takes_neighbours(bits):
    at, tensors = 0x7000_0000_0000, []
    for count in (1, 255, 4096, 4097, 0, 12288):
        t, at = _tensor(at, count, bits)
        tensors.append(t)
    assert _plan(tensors, bits) == (0, 1 + 1 + 4 + 5 + 0 + 12)                # few elements: 1024 to a workgroup
    many, at = _tensor(at, 5000 * 1024 + 1, bits)
    assert _plan(tensors + [many], bits) == (0, 1 + 1 + 1 + 2 + 0 + 3 + 1251)  # many: 4096


def test_plan_refusals():
    a, at = _tensor(0x7000_0000_0000, 1000)
    b, _ = _tensor(at, 512)
    assert _plan([a, b])[0] == 0
    assert _plan([a, a])[0] == OVERLAP                                       # the same tensor twice
    assert _plan([a], nbytes=32)[0] == WORKSPACE
    for change, status in [(dict(param=None), NULL), (dict(grad=None), NULL), (dict(first=None), NULL), (dict(copy=None), NULL),
                           (dict(param=a.param + 4), ALIGN), (dict(copy=a.copy + 2), ALIGN),
                           (dict(param=a.param + 16 * 100), OVERLAP),        # runs into another tensor's buffers
                           (dict(grad=a.param), OVERLAP), (dict(count=-1), VALUE), (dict(count=(1 << 40) + 1), VALUE)]:
        c = B.AdamWTensor(*[getattr(b, f) for f, _ in B.AdamWTensor._fields_])
        for k, v in change.items():
            setattr(c, k, v)
        assert _plan([a, c])[0] == status, change
    shared = B.AdamWTensor(*[getattr(b, f) for f, _ in B.AdamWTensor._fields_])
    shared.grad = a.grad                                                     # (a gradient read twice is harmless)
    assert _plan([a, shared])[0] == 0
    for kw in (dict(bits=16), dict(grad=3), dict(copy=2), dict(copy=-2)):
        assert _plan([a], **kw)[0] == VALUE
    assert _plan([a], bits=8)[0] == NULL                                     # no scales
    assert B.lib().fp6_adamw_plan_bytes(None, 1) == 0


@pytest.mark.parametrize("change,status", [
    (dict(plan=None), NULL), (dict(step=None), NULL), (dict(options=None), NULL), (dict(bits=4), VALUE), (dict(items=-1), VALUE),
    (dict(beta1=1.0), VALUE), (dict(beta2=-0.1), VALUE), (dict(eps=float("nan")), VALUE), (dict(lr=-1.0), VALUE),
    (dict(lr=float("inf")), VALUE), (dict(weight_decay=-1e-3), VALUE), (dict(plan=0x7000_0000_0008), ALIGN),
    (dict(step=0x7000_0000_0002), ALIGN), (dict(lr_device=0x7000_0000_0001), ALIGN),
])
def test_step_refusals(change, status):
    a = _addresses(2)
    c = dict(plan=a[0], items=1, bits=32, grad=2, copy=-1, step=a[1], lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0,
             lr_device=None)
    c.update(change)
    o = B.AdamWOptions(c["lr"], c["beta1"], c["beta2"], c["eps"], c["weight_decay"], c["lr_device"], None, None, 0)
    o = None if "options" in change else ctypes.byref(o)
    assert B.lib().fp6_adamw(c["plan"], c["items"], c["bits"], c["grad"], c["copy"], c["step"], o, None) == status


def test_no_cpu_path():
    X, A, Bm, Y = torch.zeros(2, 64).half(), torch.zeros(1, 8, 64).half(), torch.zeros(1, 64, 8).half(), torch.zeros(2, 64).half()
    with pytest.raises(P.Fp6Error, match="GPU"):
        P.fp6_lora(X, A, Bm, Y)
    with pytest.raises(P.Fp6Error, match="GPU"):
        P.fp6_lora_group([(X, A, Bm, Y)])
    with pytest.raises(P.Fp6Error, match="GPU"):
        P.fp6_lora_backward(Y, X, torch.zeros(2, 8), A, Bm)
    with pytest.raises(P.Fp6Error, match="GPU"):
        P.fp6_linear_grad(Y, Y, Y, Y, Y, 64, 64)
    with pytest.raises(P.Fp6Error, match="GPU"):
        P.fp6_adamw_plan([torch.zeros(4)], [torch.zeros(4)], [torch.zeros(4)], [torch.zeros(4)])
    with pytest.raises(P.Fp6Error, match="equally many"):
        P.fp6_adamw_plan([], [], [], [])
    with pytest.raises(P.Fp6Error, match="scales"):
        P.fp6_adamw_plan(*[[torch.zeros(4)]] * 4, first_scales=[torch.zeros(1)], second_scales=[torch.zeros(1)])
