"""The native marshalling of the calls around the frozen layer against the Python routines behind it: what it takes gives the same bits and
the same objects, what it must not take it leaves to them."""
import pytest
import torch

import paper_2312_08583_amd as P
from paper_2312_08583_amd import binding as B
from adapters_ref import adapters, normal

F16 = torch.float16


def test_host_tensors_and_other_arguments_are_left_alone():
    B.lib()
    x = torch.zeros(2, 64, dtype=F16)
    for name, n in (("lora", 9), ("lora_group", 5), ("lora_backward", 13), ("linear_grad", 10), ("adamw", 14)):
        call = B._native[name]
        for args in [(), (x,) * n, (None,) * n, (0,) * n, ([x],) * n, (x,) * (n + 1)]:
            assert call(*args) is None, (name, len(args))


def _calls(dtype):
    M, N, K, r, L = 5, 128, 192, 16, 3
    X, Y, dY = normal((M, K), 1, dtype), normal((M, N), 2, dtype), normal((M, N), 3, dtype)
    A, Bm = adapters(L, r, N, K, 4, dtype)
    index, scaling = torch.tensor([0, 2, -1, 1, 2], dtype=torch.int32, device="cuda"), torch.rand(L, device="cuda")
    hidden = normal((M, r), 6)
    ws = P.new_workspace(16 << 20, "cuda")
    W = normal((N, K), 7, F16, 0.02)
    form = P.FP6_FORMAT_E3M2_V2_BF16 if dtype == torch.bfloat16 else P.FP6_FORMAT_E3M2
    planes = P.fp6_transpose_pack(*(P.fp6_quantize_pack_v2 if dtype == torch.bfloat16 else P.fp6_quantize_pack)(W), N, K, format=form)

    def lora():
        h, out = torch.empty_like(hidden), torch.empty_like(Y)
        assert P.fp6_lora(X, A, Bm, Y, index, scaling, hidden=h, out=out, workspace=ws) is out
        into = Y.clone()
        assert P.fp6_lora(X, A, Bm, into, workspace=ws) is into
        return [out, h, into]

    def group():
        outs = [torch.empty_like(Y) for _ in range(2)]
        got = P.fp6_lora_group([(X, A, Bm, Y)] * 2, index, scaling, outs=outs, workspace=ws)
        assert isinstance(got, list) and all(g is o for g, o in zip(got, outs))
        return got

    def backward():
        dX, dA, dB = normal((M, K), 8, dtype), normal(A.shape, 9), normal(Bm.shape, 10)
        got = P.fp6_lora_backward(dY, X, hidden, A, Bm, dX, index, scaling, dA=dA, dB=dB, accumulate=True, workspace=ws)
        assert isinstance(got, tuple) and got[0] is dX and got[1] is dA and got[2] is dB
        none = P.fp6_lora_backward(dY, X, hidden, A, Bm, dA=torch.empty_like(dA), dB=torch.empty_like(dB), workspace=ws)
        assert none[0] is None
        return list(got) + list(none[1:])

    def grad():
        out = torch.empty_like(X)
        assert P.fp6_linear_grad(dY, *planes, N, K, format=form, out=out, workspace=ws) is out
        return [out]

    def adamw():
        p, g, m, v = (normal((300,), 20 + i).abs() for i in range(4))
        plan, step = P.fp6_adamw_plan([p], [g], [m], [v]), torch.zeros(1, dtype=torch.int32, device="cuda")
        assert P.fp6_adamw(plan, step, 1e-3, 0.9, 0.99, 1e-8, 0.1, grad_scale=torch.ones(1, device="cuda"), seed=3) is None
        P.fp6_adamw(plan, step, torch.tensor([1e-2], device="cuda"), found_inf=torch.zeros(1, device="cuda"), seed=-1)
        return [p, m, v, step]

    return {"lora": lora, "lora_group": group, "lora_backward": backward, "linear_grad": grad, "adamw": adamw}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F16, torch.bfloat16], ids=["fp16", "bf16"])
def test_same_results_as_the_python_routines_and_plain_calls_are_taken(dtype, monkeypatch):
    for name, call in _calls(dtype).items():
        native, taken = B._native[name], []
        monkeypatch.setitem(B._native, name, lambda *a: taken.append(native(*a)) or taken[-1])
        fast = call()
        assert taken and all(t is not None for t in taken), name
        monkeypatch.setitem(B._native, name, B._not_loaded)
        for f, s in zip(fast, call()):
            assert f.dtype == s.dtype and torch.equal(f.view(torch.int8), s.view(torch.int8)), name
        monkeypatch.setitem(B._native, name, native)


@pytest.mark.gpu
def test_errors_are_the_librarys():
    X, Y = normal((4, 64), 1, F16), normal((4, 64), 2, F16)
    A, Bm = adapters(1, 8, 64, 64, 3, F16)
    ws = P.new_workspace(16 << 20, "cuda")
    with pytest.raises(P.Fp6Error, match="overlaps"):
        P.fp6_lora(X, A, Bm, Y, out=X, workspace=ws)
    with pytest.raises(P.Fp6Error, match="workspace"):
        P.fp6_lora(X, A, Bm, Y, workspace=ws[:256])
    with pytest.raises(P.Fp6Error, match="outside"):
        P.fp6_lora(X, A[:, :4].contiguous(), Bm[:, :, :4].contiguous(), Y, workspace=ws)
    p = [torch.zeros(8, device="cuda") for _ in range(4)]
    with pytest.raises(P.Fp6Error, match="outside"):
        P.fp6_adamw(P.fp6_adamw_plan(*[[x] for x in p]), torch.zeros(1, dtype=torch.int32, device="cuda"), 1e-3, 1.0)


@pytest.mark.gpu
def test_other_tensors_are_left_to_the_python_routines():
    X, Y = normal((4, 64), 1, F16), normal((4, 64), 2, F16)
    A, Bm = adapters(1, 8, 64, 64, 3, F16)
    ws = P.new_workspace(16 << 20, "cuda")
    native = B._native["lora"]
    assert native(X, A, Bm, Y, None, None, None, torch.empty_like(Y), ws) is not None

    class Sub(torch.Tensor):
        pass

    for args in [(X.float(), A, Bm, Y), (X, A.float(), Bm, Y), (X.as_subclass(Sub), A, Bm, Y), (X, A, Bm, Y[:3]), (X.cpu(), A, Bm, Y),
                 (X, A[0], Bm, Y), (X, A, Bm.transpose(1, 2), Y)]:
        assert native(*args, None, None, None, None, ws) is None
    assert native(X, A, Bm, Y, torch.zeros(4, device="cuda"), None, None, None, ws) is None
    assert native(X, A, Bm, Y, None, None, None, None, None) is None
    # parameters are plain tensors
    out = P.fp6_lora(X, torch.nn.Parameter(A), torch.nn.Parameter(Bm), Y, out=torch.empty_like(Y), workspace=ws)
    assert torch.equal(out, P.fp6_lora(X, A, Bm, Y, out=torch.empty_like(Y), workspace=ws))
