"""GPU: the tensors of a group's list live until the call is done, whatever another thread does to the list meanwhile.  The entry points are exchanged
for ones that empty the list in place of launching anything."""
import ctypes
import gc
import weakref

import pytest
import torch

import paper_2312_08583_amd as P
from paper_2312_08583_amd import binding as B
from paper_2312_08583_amd import build as hip_build

pytestmark = pytest.mark.gpu
F16 = torch.float16


def _lora_layers():
    return [(torch.zeros(4, 64, dtype=F16, device="cuda"), torch.zeros(2, 8, 64, dtype=F16, device="cuda"),
             torch.zeros(2, 128, 8, dtype=F16, device="cuda"), torch.zeros(4, 128, dtype=F16, device="cuda")) for _ in range(2)]


def _linear_layers():
    return [(torch.zeros(4, 64, dtype=F16, device="cuda"), torch.zeros(128 * 32, dtype=torch.uint8, device="cuda"),
             torch.zeros(128 * 16, dtype=torch.uint8, device="cuda"), torch.zeros(128, dtype=F16, device="cuda"), 128, 64) for _ in range(2)]


@pytest.fixture
def restored():
    yield
    B._bind_native(B.lib(), hip_build.native_path())


def _empties(layers, alive):
    refs = [weakref.ref(t) for layer in layers for t in layer if isinstance(t, torch.Tensor)]

    def entry(*_):
        layers.clear()
        gc.collect()
        alive.append([r() is not None for r in refs])
        return 0

    return entry, refs


@pytest.mark.parametrize("native", [True, False], ids=["native", "python"])
@pytest.mark.parametrize("adapters", [True, False], ids=["lora_group", "linear_group"])
def test_tensors_live_until_the_call_is_done(adapters, native, restored, monkeypatch):
    L, alive = B.lib(), []
    layers = _lora_layers() if adapters else _linear_layers()
    outs = None if adapters else [torch.empty(4, 128, dtype=F16, device="cuda") for _ in range(2)]
    ws = P.new_workspace(16 << 20, "cuda")
    entry, refs = _empties(layers, alive)
    name = "fp6_lora_group" if adapters else "fp6_linear_group"
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value  # noqa: E731
    if native:
        callback = ctypes.CFUNCTYPE(ctypes.c_int, *getattr(L, name).argtypes)(entry)
        module = B._native["lora_group"].__self__
        if adapters:
            module.bind_adapters(address(callback), *map(address, (L.fp6_lora_backward, L.fp6_linear_grad, L.fp6_adamw)))
        else:
            entries = [L.fp6_linear, L.fp6_linear_variant, L.fp6_linear_fgq, L.fp5_linear, L.fp6_linear_v2, L.fp6_linear_v2_bf16, callback,
                       L.fp6_linear_workspace_bytes, L.fp6_linear_variant_workspace_bytes, L.fp6_linear_fgq_workspace_bytes,
                       L.fp5_linear_workspace_bytes, L.fp6_linear_v2_workspace_bytes, L.fp6_linear_group_workspace_bytes]
            module.bind(*map(address, entries), B._check)
    else:
        monkeypatch.setattr(L, name, entry)
        monkeypatch.setitem(B._native, "lora_group", B._not_loaded)
        monkeypatch.setattr(B, "_native_group", B._not_loaded)
    results = P.fp6_lora_group(layers, workspace=ws) if adapters else P.fp6_linear_group(layers, outs=outs, workspace=ws)
    assert len(results) == 2 and not layers and len(alive) == 1 and all(alive[0]), alive
    del results
    gc.collect()
    assert not any(r() is not None for r in refs)          # and no longer
