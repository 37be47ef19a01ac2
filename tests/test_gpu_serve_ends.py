"""Products and experts with values at the ends of their range: scale codes from 0 to 253 on one side or both, sums down to bf16's subnormals, activations far from one.

Beside the bounds of serve_reference a result below bf16's normal range is off by half a step of its subnormals, 2^-134, and an fp32 sum there by 2^-149 for each of its at most 2^12 terms:
2^-133 together."""
import pytest
import torch

import serve_reference as ref
from paper_2503_16672_amd import serve

BF16 = torch.bfloat16
pytestmark = pytest.mark.gpu


def _normal(shape, seed, scale):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(BF16).cuda()


def _holds(got, y, d):
    return bool(((got.double() - y).abs() <= d + ref.U * (y.abs() + d) + 2.0 ** -133).all())


# (few tokens in each form, the GEMM)
@pytest.mark.parametrize("T,K,N", [(3, 160, 72), (20, 544, 264), (70, 160, 264), (300, 1024, 512)])
@pytest.mark.parametrize("x,w", [(-100, 100), (-126, 120), (-128, 125), (-131, 125), (120, -126), (125, -131), (-60, -60), (60, 60), (-70, -56), (-63, -63), (-66, -66)])
def test_products(T, K, N, x, w):
    X, W = _normal((T, K), 1, 2.0 ** x), _normal((K, N), 2, 2.0 ** w)
    assert _holds(serve.linear_mx4(X, serve.Mx4Weight(W)), *ref.product(ref.values(X), ref.values(W, 0)))


@pytest.mark.parametrize("weights", ["bf16", "mx4"])
@pytest.mark.parametrize("T", [1, 5, 40])
@pytest.mark.parametrize("x,up,down", [(-60, 60, 0), (50, -50, 100), (-100, 100, -50), (0, -60, 100), (-20, -20, 60), (0, 0, -120)])
def test_experts(T, x, up, down, weights):
    D, F, E, k = 128, 192, 9, 3
    X, Wr, Wgu, Wd = (_normal(s, i, a) for i, (s, a) in enumerate((((T, D), 2.0 ** x), ((D, E), 0.1 * 2.0 ** -x), ((E, D, 2 * F), 0.1 * 2.0 ** up), ((E, F, D), 0.1 * 2.0 ** down))))
    Y = serve.MoeContext(T, Wr, Wgu, Wd, k, weights=weights).fwd(X)
    assert _holds(Y, *ref.moe(X, Wr, Wgu, Wd, k, "silu", True, weights == "mx4"))
