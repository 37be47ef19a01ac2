"""Gates as large as the element type takes them: a(G) is G or 0, in every forward kernel of the gated block (bf16: GEMM core and few tokens; int8: the same two)."""
import pytest
import torch

from paper_2503_16672_amd import block

D = F = 64
VALUES = [2e4, 2e19, 3e38]


@pytest.mark.gpu
@pytest.mark.parametrize("v", VALUES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,training", [(5, False), (64, False), (64, True)])
def test_large_gates(T, training, act, v):
    """Token t has the one gate value +-v everywhere, U = 1 and Wd = 1: a single product each, so Y is exact."""
    X = torch.eye(T, D, dtype=torch.bfloat16, device="cuda")
    Wgu = torch.ones((D, 2 * F), dtype=torch.bfloat16, device="cuda")
    Wgu[:, :F] = torch.where(torch.arange(D, device="cuda") % 2 == 0, v, -v)[:, None]
    Wd = torch.eye(F, dtype=torch.bfloat16, device="cuda")
    ctx = block.GatedContext(T, D, F, act=act, training=training)
    assert torch.equal(ctx.fwd(X, Wgu, Wd), Wgu[:T, :F].clamp(min=0))
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,training", [(5, False), (64, False), (64, True)])
def test_infinite_gates(T, training, act):
    """a(infinity) = infinity: gates that overflow as sums of 64 products of 3e38."""
    X, Wgu, Wd = (torch.ones(s, dtype=torch.bfloat16, device="cuda") for s in ((T, D), (D, 2 * F), (F, D)))
    Wgu[:, :F] = 3e38
    ctx = block.GatedContext(T, D, F, act=act, training=training)
    assert bool((ctx.fwd(X, Wgu, Wd) == float("inf")).all())
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("v", VALUES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T", [5, 64])
def test_large_gates_in_int8(T, act, v):
    """Feature f has the gate +-v for every token.  Codes are 127 or 0; what is rounded are the scales (fp32: 2^-20 is more than all of them), h (bf16, less than half a code) and Y
    (bf16: 2^-8 of it at most)."""
    X = torch.zeros((T, D), dtype=torch.bfloat16, device="cuda")
    X[:, 3] = 1
    Wgu = torch.ones((D, 2 * F), dtype=torch.bfloat16, device="cuda")
    Wgu[:, :F] = torch.where(torch.arange(F, device="cuda") % 2 == 0, v, -v)
    ctx = block.GatedI8Context(T, Wgu, torch.eye(F, dtype=torch.bfloat16, device="cuda"), act=act)
    Y, want = ctx.fwd(X).double(), Wgu[3, :F].clamp(min=0).double().expand(T, F)
    assert bool(((Y - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want).all())
    ctx.close()
