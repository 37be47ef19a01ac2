"""The operators around the block run on the current device: the binding refuses tensors of another one before anything is launched, and a context waits for its own."""
import ctypes

import pytest
import torch

from paper_2503_16672_amd import block

BF16, F32 = torch.bfloat16, torch.float32


def _calls(new):
    """Every call of the binding that takes tensors and no context, on tensors that `new` makes."""
    X, W, w = new((4, 64), BF16), new((64, 64), BF16), new((64,), F32)
    v = new((4,), F32)
    W8 = object.__new__(block.I8Weight)
    W8.K, W8.N, W8.data = 64, 64, new((256 * (128 + 8),), torch.uint8)
    return {"layer_norm_fwd": lambda: block.layer_norm_fwd(X, w, w, residual=X), "layer_norm_bwd": lambda: block.layer_norm_bwd(X, X, w, v, v, dS=X),
            "I8Weight": lambda: block.I8Weight(W), "quantise_i8": lambda: block.quantise_i8(X), "linear_i8": lambda: block.linear_i8(X, W8),
            "matmul_i8": lambda: block.matmul_i8(new((4, 64), torch.int8), v, W8)}


NAMES = ("layer_norm_fwd", "layer_norm_bwd", "I8Weight", "quantise_i8", "linear_i8", "matmul_i8")


class _Lib:
    """Stands in for the library: sizes, and a note of what was launched."""

    def __init__(self):
        self.launched = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith(("_scratch", "_bytes")):
                return 64
            self.launched.append(name)
            return 0
        return call


class _Elsewhere(torch.Tensor):
    """A tensor that says it is on GPU 1."""
    is_cuda = True
    device = torch.device("cuda", 1)

    def get_device(self):
        return 1

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        with torch._C.DisableTorchFunctionSubclass():
            return func(*args, **(kwargs or {}))


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_another_device_are_refused(name, monkeypatch):
    lib = _Lib()
    monkeypatch.setattr(block, "lib", lambda: lib)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    empty, empty_like = torch.empty, torch.empty_like
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **k: empty(*a, **k).as_subclass(_Elsewhere))
    monkeypatch.setattr(torch, "empty_like", lambda t: empty_like(t).as_subclass(_Elsewhere))
    call = _calls(lambda shape, dtype: torch.zeros(shape, dtype=dtype).as_subclass(_Elsewhere))[name]
    with pytest.raises(ValueError, match="device"):
        call()
    assert not lib.launched


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
    X, Wgu, Wd = (torch.ones(s, dtype=BF16, device="cuda") for s in ((4, 64), (64, 128), (64, 64)))
    bf16, i8 = block.GatedContext(4, 64, 64, training=True), block.GatedI8Context(4, Wgu, Wd)
    bf16.fwd(X, Wgu, Wd)
    torch.cuda.synchronize()
    with monkeypatch.context() as m:
        m.setattr(torch._C, "_cuda_getDevice", lambda: 1)
        for call in (lambda: bf16.fwd(X, Wgu, Wd), lambda: bf16.bwd(X, X, Wgu, Wd), lambda: i8.set_weights(Wgu, Wd), lambda: i8.fwd(X)):
            with pytest.raises(ValueError, match="device"):
                call()


def test_a_context_waits_for_its_own_device(monkeypatch):
    waited, lib = [], _Lib()
    monkeypatch.setattr(block, "lib", lambda: lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: waited.append(device))

    def create(out, *args):
        ctypes.cast(out, ctypes.POINTER(ctypes.c_void_p))[0] = 0x1000
        return 0
    lib.gated_ctx_create = create
    ctx = block.GatedContext(4, 64, 64)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    ctx.close()
    assert waited == [1] and lib.launched == ["gated_ctx_destroy"]
