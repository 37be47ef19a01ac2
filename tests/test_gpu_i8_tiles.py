"""int8 products on the GEMM core's larger tiles (256 x 256, 256 x 128; tests/test_block_rules.py holds that these sizes take them), which the sizes of test_gpu_i8.py do
not reach.  Definitions and tolerances are that file's."""
import pytest
import torch

from paper_2503_16672_amd import block
from test_gpu_i8 import U, _act, _normal, _product, _quantise

PRODUCTS = [(2990, 4160, 4168), (3499, 2112, 2184)]
GATED = [(2990, 4160, 4160), (3499, 2112, 2112), (1801, 2112, 2112)]


@pytest.mark.gpu
@pytest.mark.parametrize("T,K,N", PRODUCTS)
def test_product(T, K, N):
    X, W = _normal((T, K), T), _normal((K, N), N, K ** -0.5)
    x8, sx = _quantise(X, 1)
    w8, sw = _quantise(W, 0)
    want = _product(x8.cuda(), sx.cuda(), w8.cuda(), sw.cuda())
    W8 = block.I8Weight(W.cuda())
    assert torch.equal(block.linear_i8(X.cuda(), W8), want)
    assert torch.equal(block.matmul_i8(*block.quantise_i8(X.cuda()), W8), want)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,D,F", GATED)
def test_gated_block(T, D, F, act):
    X, Wgu, Wd = _normal((T, D), 1).cuda(), _normal((D, 2 * F), 2, D ** -0.5).cuda(), _normal((F, D), 3, F ** -0.5).cuda()
    ctx = block.GatedI8Context(T + 250, Wgu, Wd, act=act)
    ctx.fwd(_normal((T + 250, D), 4, 100.0).cuda())
    Y = ctx.fwd(X)
    (x8, sx), (w8, sw), (d8, sd) = _quantise(X, 1), _quantise(Wgu, 0), _quantise(Wd, 0)
    gu = (x8.double() @ w8.double()) * sx.double() * sw.double()
    h = _act(gu[:, :F], act) * gu[:, F:]
    top = h.abs().amax(dim=1, keepdim=True).float()
    sh = torch.where(top > 0, top * (1.0 / 127.0), torch.ones_like(top))
    h8 = torch.round(h.to(torch.bfloat16).float() / sh).clamp(-127, 127)
    W = d8.double() * sd.double()
    ref = (h8.double() @ W) * sh.double()
    sigma = torch.sqrt((U * ref) ** 2 / 3 + 2.0 ** -12 * sh.double() ** 2 * (W ** 2).sum(0))
    err = (Y.double() - ref).abs()
    assert bool((err <= 7 * sigma + 2 * sh.double() * W.abs().amax(0)).all()), float((err / sigma).max())
    assert float(err.norm()) <= 1.1 * float(sigma.norm())
    assert torch.equal(ctx.fwd(X[T - 16:].contiguous()), Y[T - 16:])      # (the kernels for few tokens)
    ctx.close()
