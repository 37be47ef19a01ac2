"""mx4 numbers bit for bit against the definition, products and the gated block on them within the bounds of serve_reference."""
import ctypes

import pytest
import torch

import serve_reference as ref
from paper_2503_16672_amd import serve
from paper_2503_16672_amd.ffn24 import Ffn24Error

BF16, F32 = torch.bfloat16, torch.float32
pytestmark = pytest.mark.gpu


def _normal(shape, seed, scale=1.0, dtype=BF16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def _check_codes(X):
    codes, scales = serve.quantise_mx4(X)
    want, s, v = ref.mx4(X)
    assert torch.equal(scales.long(), s)
    good = (s != 255).repeat_interleave(32, dim=1)
    assert bool((ref.unpack(codes) == want)[good].all())
    for dtype in (BF16, F32):
        back = serve.dequantise_mx4(codes, scales, dtype=dtype)
        assert back.dtype == dtype and torch.equal(torch.isnan(back), ~good) and torch.equal(back.double()[good], v[good])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,K", [(1, 32), (1, 1024), (3, 96), (7, 4128), (333, 1088), (2, 131072), (1000, 4096)])
def test_codes_and_values(T, K, dtype):
    X = _normal((T, K), T + K, dtype=dtype)
    X[T - 1, K // 2:] = 0
    _check_codes(X * torch.exp2(torch.randint(-6, 6, (K,), generator=torch.Generator().manual_seed(1)).cuda()).to(dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_borders_and_the_ends_of_the_range(dtype):
    """Every border between neighbours and its neighbours in the type, at scales from the least to the largest; zeros of both signs, subnormals, infinities, NaN."""
    rows = []
    eps = torch.finfo(dtype).eps
    points = [s * b * f for b in (0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.0) for f in (1 - eps, 1.0, 1 + eps) for s in (1, -1)]
    for e in (-149, -140, -130, -128, -127, -126, -100, -3, 0, 3, 100, 124, 125):
        for i in range(0, len(points), 31):
            part = points[i:i + 31]
            rows.append([m * 2.0 ** e for m in [4.0, *part, *[0.0] * (31 - len(part))]])
    big = float(torch.finfo(dtype).max)
    rows += [[big] * 32, [-0.0] * 32, [-0.0, big] + [1.0] * 30, [float("inf")] + [1.0] * 31, [1.0] * 31 + [float("nan")], [-float("inf")] * 32]
    X = torch.tensor(rows, dtype=torch.float64).to(dtype).cuda()
    _check_codes(X)
    _check_codes(X.reshape(1, -1)[:, :X.numel() // 64 * 64].reshape(-1, 64).contiguous())


def test_values_of_all_codes():
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(16)[None].repeat(256, 1).contiguous()
    scales = torch.arange(256, dtype=torch.uint8, device="cuda")[:, None].repeat(1, codes.shape[1] // 16).contiguous()
    want = ref.decode(ref.unpack(codes), scales)
    for dtype in (BF16, F32):
        got = serve.dequantise_mx4(codes, scales, dtype=dtype)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        ok = ~torch.isnan(want)
        held = want.to(dtype)                                     # (6 x 2^127 is beyond both types)
        assert torch.equal(got[ok], held[ok])


# few tokens in each kernel and form, the GEMM's tiles (tests/test_serve_rules.py), k and channels that end inside a step, a block of 64 and a tile, reductions that are split
PRODUCTS = [(1, 32, 8), (1, 2048, 520), (3, 96, 24), (16, 160, 264), (17, 544, 264), (32, 1088, 1000), (33, 1088, 1000), (64, 128, 72), (65, 224, 256), (333, 1088, 4168),
            (1000, 640, 3000), (1500, 512, 2048), (4099, 288, 4104), (2, 16416, 16), (1, 512, 16400), (13, 384, 33000), (29, 8224, 200), (100, 16384, 512), (130, 8992, 136),
            (48, 131072, 8), (5, 131072, 40), (9, 1024, 9000), (9, 4096, 8200), (16, 4224, 8200), (16, 4224, 33000), (2100, 3008, 5000), (4096, 16384, 4096), (2000, 4096, 8200),
            (3, 32, 1 << 20), (40, 64, 1 << 20), (1 << 20, 32, 8), (1 << 20, 96, 136), (3, 131072, 2048)]


@pytest.mark.parametrize("T,K,N", PRODUCTS)
def test_product(T, K, N):
    X, W = _normal((T, K), T), _normal((K, N), N, K ** -0.5)
    W[:, N - 1] = 0
    W4 = serve.Mx4Weight(W)
    Y = serve.linear_mx4(X, W4)
    y, d = ref.product(ref.values(X), ref.values(W, 0))
    assert ref.holds(Y, y, d), (T, K, N, float(((Y.double() - y).abs() - d).max()))
    assert bool((Y[:, N - 1] == 0).all())
    codes, scales = serve.quantise_mx4(W.T.contiguous())
    assert torch.equal(serve.linear_mx4(X, serve.Mx4Weight.from_codes(codes, scales)), Y)


@pytest.mark.parametrize("T,K,N", [(4, 160, 40), (20, 544, 264), (70, 160, 264), (300, 4096, 512)])
def test_tokens_and_channels_are_apart(T, K, N):
    """A token with a NaN or an infinity does not reach another one, nor a channel with one."""
    X, W = _normal((T, K), 1), _normal((K, N), 2)
    Y = serve.linear_mx4(X, serve.Mx4Weight(W))
    X2, W2 = X.clone(), W.clone()
    X2[1, 0], X2[3, K - 1], W2[K - 1, 5] = float("nan"), float("inf"), float("nan")
    Y2 = serve.linear_mx4(X2, serve.Mx4Weight(W2))
    rows, cols = [t for t in range(T) if t not in (1, 3)], [n for n in range(N) if n != 5]
    assert torch.equal(Y2[rows][:, cols], Y[rows][:, cols]) and bool(Y2[[1, 3]].isnan().all()) and bool(Y2[:, 5].isnan().all())


def _gated(T, D, F, act, seed=1):
    X, Wgu, Wd = _normal((T, D), seed), _normal((D, 2 * F), seed + 1, D ** -0.5), _normal((F, D), seed + 2, F ** -0.5)
    return X, Wgu, Wd, ref.gated_mx4(ref.values(X), ref.values(Wgu, 0), ref.values(Wd, 0), act)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,D,F", [(1, 64, 64), (2, 128, 192), (16, 576, 1344), (17, 64, 448), (33, 192, 448), (64, 512, 2048), (65, 256, 512), (24, 2048, 4160), (4, 3968, 16384),
                                   (700, 320, 704), (1609, 640, 640), (2500, 512, 2816), (40, 1024, 8192), (12, 8192, 512), (16, 4160, 16384), (3000, 1024, 4096), (2000, 4096, 4160),
                                   (4096, 8192, 2048), (4096, 16384, 2048), (3, 131072, 64), (3, 64, 131072), (70, 64, 131072), (70, 131072, 64), (1 << 18, 64, 128)])
def test_gated_block(T, D, F, act):
    X, Wgu, Wd, (y, d) = _gated(T, D, F, act)
    ctx = serve.GatedMx4Context(T + 5, Wgu, Wd, act=act)
    Y = ctx.fwd(X)
    assert ref.holds(Y, y, d), (T, D, F, float(((Y.double() - y).abs() / (d + ref.U * y.abs())).max()))
    part = ctx.fwd(X[:(T + 1) // 2].contiguous())
    assert ref.holds(part, y[:(T + 1) // 2], d[:(T + 1) // 2])
    assert torch.equal(ctx.fwd(X), Y)                            # (results repeat)
    # other weights in the same context
    X, Wgu, Wd, (y, d) = _gated(T, D, F, act, seed=11)
    ctx.set_weights(Wgu, Wd)
    assert ref.holds(ctx.fwd(X), y, d)
    ctx.close()


def test_gated_tokens_are_apart():
    for T, D, F in [(5, 192, 320), (20, 192, 320), (100, 192, 320)]:
        X, Wgu, Wd, _ = _gated(T, D, F, "silu")
        ctx = serve.GatedMx4Context(T, Wgu, Wd)
        Y = ctx.fwd(X)
        X2 = X.clone()
        X2[2, 7] = float("nan")
        Y2 = ctx.fwd(X2)
        rows = [t for t in range(T) if t != 2]
        assert bool(Y2[2].isnan().all()) and torch.equal(Y2[rows], Y[rows])
        assert torch.equal(ctx.fwd(X), Y)                        # (and nothing of it is left in the context)


def test_streams_graphs_and_no_tokens():
    X, Wgu, Wd, (y, d) = _gated(40, 512, 1408, "gelu")
    ctx = serve.GatedMx4Context(64, Wgu, Wd, act="gelu")
    W4 = serve.Mx4Weight(Wd)
    H = _normal((40, 1408), 9)
    Y, Z, Yc, Zc = torch.empty_like(X), torch.empty_like(X), torch.empty_like(X), torch.empty_like(X)
    codes, scales, back = (torch.empty(s, dtype=t, device="cuda") for s, t in (((40, 256), torch.uint8), ((40, 16), torch.uint8), ((40, 512), BF16)))

    def work(y, z):
        ctx.fwd(X, Y=y)
        serve.linear_mx4(H, W4, Y=z)
        serve.quantise_mx4(y, codes=codes, scales=scales)
        serve.dequantise_mx4(codes, scales, Y=back)

    work(Y, Z)
    want = back.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        work(Yc, Zc)
    torch.cuda.synchronize()
    assert torch.equal(Y, Yc) and torch.equal(Z, Zc) and ref.holds(Y, y, d)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        work(Yc, Zc)
    for i in range(4):
        keep = X.clone()
        X.mul_(-1 if i % 2 else 1)
        work(Y, Z)
        want = back.clone()
        for t in (Yc, Zc, back):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, Yc) and torch.equal(Z, Zc) and torch.equal(back, want)
        X.copy_(keep)
    empty = X[:0]
    assert ctx.fwd(empty).shape == (0, 512) and serve.linear_mx4(H[:0], W4).shape == (0, 512)
    codes, scales = serve.quantise_mx4(empty)
    assert serve.dequantise_mx4(codes, scales).shape == (0, 512)


def test_refusals():
    X, W = _normal((4, 64), 1), _normal((64, 128), 2)
    W4 = serve.Mx4Weight(W)
    ctx = serve.GatedMx4Context(4, W, _normal((64, 64), 3))
    for call in (lambda: serve.quantise_mx4(X[:, :48]), lambda: serve.quantise_mx4(X[:, :32]), lambda: serve.quantise_mx4(X.half()), lambda: serve.linear_mx4(X[:, :32].contiguous(), W4),
                 lambda: serve.linear_mx4(X.float(), W4), lambda: ctx.fwd(X.float()), lambda: ctx.fwd(_normal((4, 128), 1)), lambda: serve.GatedMx4Context(4, W, W, act="relu"),
                 lambda: serve.GatedMx4Context(4, W, W), lambda: serve.dequantise_mx4(torch.zeros((2, 32), dtype=torch.uint8, device="cuda"), torch.zeros((2, 1), dtype=torch.uint8, device="cuda")),
                 lambda: serve.dequantise_mx4(*serve.quantise_mx4(X), dtype=torch.float16), lambda: serve.Mx4Weight(W.float())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ctx.fwd(_normal((5, 64), 1)), lambda: serve.Mx4Weight(_normal((64, 12), 1)), lambda: serve.Mx4Weight(_normal((48, 16), 1)),
                 lambda: serve.GatedMx4Context(4, _normal((96, 128), 1), _normal((64, 96), 1)), lambda: serve.GatedMx4Context(0, W, _normal((64, 64), 3))):
        with pytest.raises(Ffn24Error):
            call()
    h = ctypes.c_void_p()
    L = serve.lib()
    assert L.gated_mx4_ctx_create(ctypes.byref(h), 4, 64, 64, 0) == 0
    assert L.gated_mx4_fwd(h, X.data_ptr(), 4, torch.empty_like(X).data_ptr(), None) == -5    # no weights yet
    assert L.gated_mx4_ctx_destroy(h) == 0
