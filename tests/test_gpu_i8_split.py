"""The gated int8 block where the down product's reduction is split over workgroups while the hidden codes lie in panel form (tests/test_block_rules.py holds that
these sizes take that path).  The definition, and the tolerance's derivation, are those of test_gpu_i8.py."""
import pytest
import torch

from paper_2503_16672_amd import block
from test_gpu_i8 import U, _act, _normal, _quantise

# every tile a split takes, 2 to 16 parts; tokens that end anywhere in a block of 256, hidden sizes that are no multiple of 128
SIZES = [(33, 2048, 5440), (64, 4096, 16384), (128, 4096, 12288), (200, 5120, 13824), (20, 1280, 5120), (300, 512, 8256), (90, 4096, 16448), (1097, 1024, 14976), (700, 320, 16384),
         (40, 64, 16384)]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,D,F", SIZES)
def test_split_down_product(T, D, F, act):
    X, Wgu, Wd = _normal((T, D), 1).cuda(), _normal((D, 2 * F), 2, D ** -0.5).cuda(), _normal((F, D), 3, F ** -0.5).cuda()
    ctx = block.GatedI8Context(T + 250, Wgu, Wd, act=act)
    ctx.fwd(_normal((T + 250, D), 4, 100.0).cuda())          # (the workspace holds other tokens' codes beyond T)
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
    # the kernels for few tokens, which have no panel form: the same bits
    few = 16
    for t in (0, T - few):
        assert torch.equal(ctx.fwd(X[t:t + few].contiguous()), Y[t:t + few])
    ctx.close()


ROWS = (2048, 8192, (1, 16, 24, 40, 100, 1000))


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_a_token_has_the_same_result_in_any_company(act):
    D, F, counts = ROWS
    X, Wgu, Wd = _normal((max(counts), D), 5).cuda(), _normal((D, 2 * F), 6, D ** -0.5).cuda(), _normal((F, D), 7, F ** -0.5).cuda()
    ctx = block.GatedI8Context(max(counts), Wgu, Wd, act=act)
    whole = ctx.fwd(X)
    for T in counts:
        assert torch.equal(ctx.fwd(X[:T].contiguous()), whole[:T]), T
    ctx.close()
