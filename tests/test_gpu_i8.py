"""Products of 8-bit integers: codes, scales and results bit for bit against the definition (the sums are whole numbers, the two roundings behind them IEEE), and the
gated block on them.

Tolerance of the gated block: its activation is computed in fp32 with a relative error below 2^-20, so one value in 2^12 may round to the other neighbour in bf16
(spacing 2^-8) and move a code by one.  sigma^2 = (2^-8 Y)^2 / 3 + 2^-12 sum_f (sh Wd)^2; an element may be off by 7 sigma and two such steps, a norm by 1.1 sigma's."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2503_16672_amd import block

U = 2.0 ** -8


def _normal(shape, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16)


def _quantise(X, dim):
    x = X.float()
    top = x.abs().amax(dim=dim, keepdim=True)
    s = torch.where(top > 0, top * (1.0 / 127.0), torch.ones_like(top))
    return torch.round(x / s).clamp(-127, 127), s


def _product(x8, sx, w8, sw):
    """fp32 rounding of the exact sum, times the product of the scales, rounded to bf16"""
    acc = (x8.double() @ w8.double()).float()
    return (acc * (sx * sw)).to(torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("T,K", [(1, 16), (3, 48), (5, 2048), (2, 2064), (1030, 1008), (1025, 2032), (1024, 4096), (7, 4112), (2, 16384), (3, 16400), (2, 131072)])
def test_codes_and_scales(T, K):
    X = _normal((T, K), T + K)
    X[T - 1, K // 2:] = 0
    if T > 2:
        X[1] = 0
    codes, scales = block.quantise_i8(X.cuda())
    c, s = _quantise(X, 1)
    assert torch.equal(scales.cpu(), s[:, 0]) and torch.equal(codes.cpu().float(), c)


# the GEMM core's five tiles, token counts from one, channels and reductions that end inside a tile and a stage
@pytest.mark.gpu
@pytest.mark.parametrize("T,K,N", [(1, 16, 8), (1, 2048, 520), (3, 80, 24), (17, 144, 264), (64, 1088, 1000), (65, 208, 256), (333, 1088, 4168), (1000, 640, 3000),
                                   (1500, 512, 2048), (2100, 1552, 5000), (4099, 272, 4104), (2, 16400, 16),
                                   (16, 1040, 40), (1, 16992, 264), (29, 8208, 200), (32, 8192, 16392), (5, 4112, 32768), (100, 16384, 512), (130, 8992, 136), (300, 6000, 1000)])
def test_product(T, K, N):
    X, W = _normal((T, K), T), _normal((K, N), N, K ** -0.5)
    W[:, N - 1] = 0
    x8, sx = _quantise(X, 1)
    w8, sw = _quantise(W, 0)
    want = _product(x8.cuda(), sx.cuda(), w8.cuda(), sw.cuda())
    W8 = block.I8Weight(W.cuda())
    Y = block.linear_i8(X.cuda(), W8)
    assert torch.equal(Y, want), (T, K, N, int((Y != want).sum()))
    codes, scales = block.quantise_i8(X.cuda())
    assert torch.equal(block.matmul_i8(codes, scales, W8), want)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40, 300])
def test_largest_sums_do_not_overflow(T):
    """127 x 127 x 2^17 is 1.6 % under 2^31."""
    K = 1 << 17
    X = torch.ones((T, K), dtype=torch.bfloat16, device="cuda")
    W = torch.ones((K, 8), dtype=torch.bfloat16, device="cuda")
    W[:, 4:] = -1
    Y = block.linear_i8(X, block.I8Weight(W))
    s = torch.tensor(1.0) * (1.0 / 127.0)
    want = (torch.tensor(float(127 * 127 * K)) * (s * s)).to(torch.bfloat16)
    assert bool((Y[:, :4] == want.cuda()).all()) and bool((Y[:, 4:] == -want.cuda()).all())


@pytest.mark.gpu
def test_tokens_are_apart():
    """A token with NaN or infinity does not reach another one, also where a reduction ends inside a stage (K 144)."""
    for T, K, N in [(4, 144, 40), (70, 144, 264)]:
        X, W8 = _normal((T, K), 1).cuda(), block.I8Weight(_normal((K, N), 2).cuda())
        Y = block.linear_i8(X, W8)
        X2 = X.clone()
        X2[1, 0], X2[3, 143] = float("nan"), float("inf")
        Y2 = block.linear_i8(X2, W8)
        good = [t for t in range(T) if t not in (1, 3)]
        assert torch.equal(Y2[good], Y[good]) and bool(Y2[1].isnan().all()) and not bool(Y2[3].isfinite().any())


def _act(x, act):
    c1, c3 = {"silu": (1.0, 0.0), "gelu": (1.5957691216057308, 1.5957691216057308 * 0.044715)}[act]
    return x * torch.sigmoid(c1 * x + c3 * x ** 3)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,D,F", [(1, 64, 64), (2, 128, 192), (16, 576, 1344), (33, 192, 448), (64, 512, 2048), (65, 256, 512), (24, 2048, 4160), (4, 3968, 16384), (700, 320, 704), (1609, 640, 640), (2500, 512, 2816)])
def test_gated_block(T, D, F, act):
    X, Wgu, Wd = _normal((T, D), 1).cuda(), _normal((D, 2 * F), 2, D ** -0.5).cuda(), _normal((F, D), 3, F ** -0.5).cuda()
    ctx = block.GatedI8Context(T + 5, Wgu, Wd, act=act)
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
    # fewer tokens on the same context: the same results for them (whole-number sums)
    part = ctx.fwd(X[:(T + 1) // 2].contiguous())
    assert torch.equal(part, Y[:(T + 1) // 2])
    ctx.close()


@pytest.mark.gpu
def test_weights_may_be_replaced_on_another_stream():
    D, F, T = 128, 256, 20
    a, b = ((_normal((D, 2 * F), s).cuda(), _normal((F, D), s + 1).cuda()) for s in (1, 5))
    X = _normal((T, D), 9).cuda()
    want = block.GatedI8Context(T, *b).fwd(X)
    ctx = block.GatedI8Context(T, *a)
    ctx.fwd(X)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.set_weights(*b)
        Y = ctx.fwd(X)
    side.synchronize()
    assert torch.equal(Y, want)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 300])
def test_replayed_in_a_graph(T):
    D, F = 256, 512
    X = _normal((T, D), 1).cuda()
    ctx = block.GatedI8Context(T, _normal((D, 2 * F), 2, D ** -0.5).cuda(), _normal((F, D), 3, F ** -0.5).cuda())
    W8 = block.I8Weight(_normal((D, 264), 4).cuda())
    run = lambda: (ctx.fwd(X), block.linear_i8(X, W8))
    run()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        out = run()
    for seed in range(3):
        X.copy_(_normal((T, D), 20 + seed).cuda())
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.gpu
def test_no_tokens_and_no_weights():
    W8 = block.I8Weight(_normal((64, 24), 0).cuda())
    X = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    assert block.linear_i8(X, W8).shape == (0, 24)
    h = ctypes.c_void_p()
    assert block.lib().gated_i8_ctx_create(ctypes.byref(h), 4, 64, 64, 0) == 0
    assert block.lib().gated_i8_fwd(h, 0x1000, 4, 0x1000, None) == -5 and block.lib().gated_i8_ctx_destroy(h) == 0


def test_refusals_without_a_gpu():
    L, a = block.lib(), 0x1000
    assert L.i8_weight_bytes(16, 8) == 256 * (128 + 8) and L.i8_weight_bytes(8, 8) == -1 and L.i8_weight_bytes(24, 8) == -1 and L.i8_weight_bytes(16, 4) == -1
    assert L.i8_weight_bytes((1 << 17) + 16, 8) == -1 and L.i8_weight_bytes(16, 0) == -1
    assert L.i8_weight(a, 16, 8, 1, a, None) == -2 and L.i8_weight(None, 16, 8, 0, a, None) == -1 and L.i8_weight(a + 2, 16, 8, 0, a, None) == -3
    assert L.quantise_i8(a, 1, 8, a, a, None) == -2 and L.quantise_i8(a, -1, 16, a, a, None) == -2 and L.quantise_i8(None, 1, 16, a, a, None) == -1
    assert L.quantise_i8(a, 1, 16, a + 4, a, None) == -3 and L.quantise_i8(None, 0, 16, None, None, None) == 0
    assert L.matmul_i8(a, a, 1, a, 16, 12, a, None) == -2 and L.matmul_i8(a, a, 1, None, 16, 8, a, None) == -1 and L.matmul_i8(a, a, 1, a, 16, 8, a + 2, None) == -3
    assert L.linear_i8_scratch(3, 16, 8) == 48 + 16 and L.linear_i8_scratch(-1, 16, 8) == -1 and L.linear_i8_scratch(1, 20, 8) == -1 and L.linear_i8_scratch(1, 16, 4) == -1
    assert L.linear_i8(a, 1, a, 20, 8, a, a, None) == -2 and L.linear_i8(a, 1, a, 16, 8, a, None, None) == -1 and L.linear_i8(a, 1, a, 16, 8, a, a + 1, None) == -3
    h = ctypes.c_void_p()
    assert L.gated_i8_ctx_create(ctypes.byref(h), 8, 64, 64, 3) == -4 and L.gated_i8_ctx_create(ctypes.byref(h), 8, 60, 64, 0) == -2
    assert L.gated_i8_ctx_create(ctypes.byref(h), 8, 64, (1 << 17) + 64, 0) == -2 and L.gated_i8_ctx_create(None, 8, 64, 64, 0) == -1 and h.value is None
    assert L.gated_i8_set_weights(None, a, a, None) == -1 and L.gated_i8_fwd(None, a, 1, a, None) == -1 and L.gated_i8_ctx_destroy(None) == 0


def test_binding_refuses_what_does_not_fit():
    with pytest.raises(block.Ffn24Error):
        block.I8Weight(torch.zeros((24, 8), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="dtype"):
        block.I8Weight(torch.zeros((16, 8)))
    with pytest.raises(ValueError, match="CUDA"):
        block.I8Weight(torch.zeros((16, 8), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="Wgu: shape"):
        block.GatedI8Context(4, torch.zeros((64, 64), dtype=torch.bfloat16), torch.zeros((64, 64), dtype=torch.bfloat16))
