"""The gated block's backward on the launches that the sizes of test_gpu_gated.py do not reach (tests/test_block_rules.py holds which): dX and the weight gradients in one
launch on each tile, or apart.  Definition and tolerances are that file's."""
import pytest
import torch

from paper_2503_16672_amd import block
from test_gpu_gated import _inputs, check, reference

SIZES = [(901, 5824, 960), (69, 5056, 192), (1000, 1088, 2944), (65, 192, 2752), (1713, 6976, 704), (805, 448, 4160), (1823, 192, 8128), (143, 3776, 320),
         (897, 4160, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,D,F", SIZES)
def test_gated_and_its_gradient(T, D, F, act):
    X, Wgu, Wd, dY = _inputs(T, D, F, seed=T + D + F)
    ctx = block.GatedContext(T + 3, D, F, act=act, training=True)
    Y = ctx.fwd(X, Wgu, Wd)
    grads = ctx.bwd(dY, X, Wgu, Wd)
    ref = reference(X, Wgu, Wd, dY, act)
    for name, got in zip(("Y", "dX", "dWgu", "dWd"), (Y, *grads)):
        check(got, ref[name], name)
    assert all(torch.equal(a, b) for a, b in zip(ctx.bwd(dY, X, Wgu, Wd), grads))
    ctx.close()
