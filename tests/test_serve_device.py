"""Serving with mx4 weights and with experts runs on the current device: the binding refuses tensors of another one, and host tensors, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2503_16672_amd import block, serve
from test_block_device import _Elsewhere, _Lib

BF16, U8 = torch.bfloat16, torch.uint8


def _calls(new):
    """Every call of the binding that takes tensors and no context, on tensors that `new` makes."""
    X, W, codes, scales = new((4, 64), BF16), new((64, 64), BF16), new((4, 32), U8), new((4, 2), U8)
    W4 = object.__new__(serve.Mx4Weight)
    W4.K, W4.N, W4.data = 64, 64, new((4096 + 1024,), U8)
    return {"quantise_mx4": lambda: serve.quantise_mx4(X, codes=codes, scales=scales), "dequantise_mx4": lambda: serve.dequantise_mx4(codes, scales, Y=X),
            "Mx4Weight": lambda: serve.Mx4Weight(W), "from_codes": lambda: serve.Mx4Weight.from_codes(new((64, 32), U8), new((64, 2), U8)),
            "linear_mx4": lambda: serve.linear_mx4(X, W4)}


NAMES = ("quantise_mx4", "dequantise_mx4", "Mx4Weight", "from_codes", "linear_mx4")


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_another_device_are_refused(name, monkeypatch):
    lib = _Lib()
    monkeypatch.setattr(serve, "lib", lambda: lib)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    empty, empty_like = torch.empty, torch.empty_like
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: empty(*a, **k).as_subclass(_Elsewhere))
    monkeypatch.setattr(torch, "empty_like", lambda t: empty_like(t).as_subclass(_Elsewhere))
    call = _calls(lambda shape, dtype: torch.zeros(shape, dtype=dtype).as_subclass(_Elsewhere))[name]
    with pytest.raises(ValueError, match="device"):
        call()
    assert not lib.launched


@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_are_refused(name, monkeypatch):
    lib = _Lib()
    monkeypatch.setattr(serve, "lib", lambda: lib)
    with pytest.raises(ValueError, match="CUDA"):
        _calls(lambda shape, dtype: torch.zeros(shape, dtype=dtype))[name]()
    assert not lib.launched


@pytest.mark.parametrize("make", ["gated", "moe"])
def test_a_context_waits_for_its_own_device_and_frees_itself_once(make, monkeypatch):
    waited, lib = [], _Lib()
    monkeypatch.setattr(serve, "lib", lambda: lib)
    monkeypatch.setattr(block, "lib", lambda: lib)
    monkeypatch.setattr(serve, "_stream", lambda *t: 0)
    monkeypatch.setattr(serve, "_ptr", lambda t: 0x1000)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: waited.append(device))

    def create(out, *args):
        ctypes.cast(out, ctypes.POINTER(ctypes.c_void_p))[0] = 0x1000
        return 0
    lib.gated_mx4_ctx_create = lib.moe_ctx_create = create
    z = lambda *shape: torch.zeros(shape, dtype=BF16)
    ctx = serve.GatedMx4Context(4, z(64, 128), z(64, 64)) if make == "gated" else serve.MoeContext(4, z(64, 4), z(4, 64, 128), z(4, 64, 64), 2)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    ctx.close()
    ctx.close()
    name = "gated_mx4" if make == "gated" else "moe"
    assert waited == [1] and lib.launched == [f"{name}_set_weights", f"{name}_ctx_destroy"]


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_calls_with_another_device_current_are_refused(name, monkeypatch):
    call = _calls(lambda shape, dtype: torch.ones(shape, dtype=dtype, device="cuda"))[name]
    call()
    torch.cuda.synchronize()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    with pytest.raises(ValueError, match="device"):
        call()


@pytest.mark.gpu
def test_contexts_refuse_tensors_of_another_device(monkeypatch):
    new = lambda *shape: torch.ones(shape, dtype=BF16, device="cuda")
    X, Wgu, Wd = new(4, 64), new(64, 128), new(64, 64)
    gated, moe = serve.GatedMx4Context(4, Wgu, Wd), serve.MoeContext(4, new(64, 4), new(4, 64, 128), new(4, 64, 64), 2)
    gated.fwd(X), moe.fwd(X)
    torch.cuda.synchronize()
    with monkeypatch.context() as m:
        m.setattr(torch._C, "_cuda_getDevice", lambda: 1)
        for call in (lambda: gated.fwd(X), lambda: gated.set_weights(Wgu, Wd), lambda: moe.fwd(X), lambda: moe.set_weights(new(64, 4), new(4, 64, 128), new(4, 64, 64))):
            with pytest.raises(ValueError, match="device"):
                call()
