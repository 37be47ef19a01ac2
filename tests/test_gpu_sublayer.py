"""Norm, gated block, backward of both and int8 serving together, against autograd in 64 bits over two sublayers.

Tolerances.  Every tensor handed from kernel to kernel is rounded to bf16 once, u / sqrt(3) of its norm (u = 2^-8).  Forward there are 4 of them a sublayer (sum, norm, H,
output), backward 4 more (dG | dU, dX, the two sums): at most 16 on any way through two sublayers, each of which the gate may double: 2 sqrt(16 / 3) u = 4.6 u."""
import pytest
import torch

from paper_2503_16672_amd.sublayer import GatedSublayer

U = 2.0 ** -8
pytestmark = pytest.mark.gpu


def _plain(x, stream, weights):
    w, b, Wgu, Wd = weights
    s = stream + x
    c = s - s.mean(1, keepdim=True)
    y = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * w + b
    gu = y @ Wgu
    F = Wd.shape[0]
    return (gu[:, :F] * torch.sigmoid(gu[:, :F]) * gu[:, F:]) @ Wd, s


def _inputs(T, D):
    g = torch.Generator(device="cuda").manual_seed(T)
    return [(torch.randn((T, D), generator=g, device="cuda")).to(torch.bfloat16) for _ in range(4)]


@pytest.mark.parametrize("T,D,F", [(1, 64, 128), (77, 192, 512), (600, 512, 1408)])
def test_two_sublayers(T, D, F):
    x, stream, dx, dstream = _inputs(T, D)
    layers = [GatedSublayer(T, D, F, seed=i) for i in range(2)]
    a, s = x, stream
    for layer in layers:
        a, s = layer.forward(a, s)
    da, ds, grads = dx, dstream, []
    for layer in reversed(layers):
        da, g = layer.backward(da, ds)
        ds = da
        grads = g + grads
    leaves = [t.double().requires_grad_() for t in (x, stream)]
    weights = [[t.double().requires_grad_() for t in (l.norm_weight, l.norm_bias, l.Wgu, l.Wd)] for l in layers]
    ra, rs = leaves
    for w in weights:
        ra, rs = _plain(ra, rs, w)
    ((ra * dx.double()).sum() + (rs * dstream.double()).sum()).backward()
    got = [a, s, da, *grads]
    want = [ra, rs, leaves[0].grad, *(t.grad for w in weights for t in w)]
    assert torch.equal(leaves[0].grad, leaves[1].grad)
    for i, (p, q) in enumerate(zip(got, want)):
        off, size = float((p.double() - q.detach()).norm()), float(q.detach().norm())
        assert off <= 4.6 * U * size, (i, off / size / U)


@pytest.mark.parametrize("T", [1, 16, 40, 300])
def test_serving_in_int8_is_near_bf16(T):
    """Codes are off by up to half a scale, a 254th of the row's largest value: 1 / (254 sqrt(3)) x (largest / rms) of a tensor's norm.  For the tokens and weights (largest 3-5 rms)
    0.7-1.1 %, for the activation (a product, largest up to 15 rms) 3.5 %: 6 % holds them all."""
    D, F = 512, 1408
    x, stream, _, _ = _inputs(T, D)
    layer = GatedSublayer(T, D, F)
    a, s = layer.serve(x, stream)
    b, t = layer.serve(x, stream, layer.quantised())
    assert torch.equal(s, t)
    off = float((a.double() - b.double()).norm() / a.double().norm())
    assert 1e-4 < off < 0.06, off
