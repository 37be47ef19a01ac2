"""The gated feed-forward block in bf16, forward and backward, against its definition in 64 bits.

Tolerances.  Rounding to bf16 moves a value by at most u = 2^-8 of it, u / sqrt(3) in the mean square if the error is uniform.  With independent errors an output's
deviation is sigma = u / sqrt(3) sqrt(sum over its products of (number of roundings) x product^2 + output^2): H, dU and dG
carry one rounding each.  An element may be off by 7 sigma, an output's norm by 1.1 of sigma's; the approximate
reciprocal and exponential (2^-22) vanish beside that.  Two things vanish for most elements only, and have terms of their own:
G, U and dH are sums of K products in fp32: the partial sums have k / K of the variance S^2 = sum of the products' squares, each addition rounds by 2^-24 of its
partial sum (/ sqrt(3)), together 2^-24 S sqrt(K / 6), which shows where G is next to 0 and a(G) with it;
and G, cut to 24 bits for the backward, is off by 2^-15 of it at most, which shows where the gate's slope is next to its zero (G = -0.75 or -1.28)."""
import numpy as np
import pytest
import torch

from paper_2503_16672_amd import block

U = 2.0 ** -8
ACT = {"silu": (1.0, 0.0), "gelu": (1.5957691216057308, 1.5957691216057308 * 0.044715)}


def _act(x, act):
    c1, c3 = ACT[act]
    s = torch.sigmoid(c1 * x + c3 * x ** 3)
    return x * s, s + x * s * (1 - s) * (c1 + 3 * c3 * x * x)


def _bend(x, act):
    """The derivative of the slope."""
    c1, c3 = ACT[act]
    s, p1 = torch.sigmoid(c1 * x + c3 * x ** 3), c1 + 3 * c3 * x * x
    s1 = s * (1 - s) * p1
    return 2 * s1 + x * (s1 * (1 - 2 * s) * p1 + s * (1 - s) * 6 * c3 * x)


def _inputs(T, D, F, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda s, scale=1.0: (torch.randn(s, generator=g, device="cuda") * scale).to(torch.bfloat16)
    return n((T, D)), n((D, 2 * F), D ** -0.5), n((F, D), F ** -0.5), n((T, D))


def reference(X, Wgu, Wd, dY, act):
    """Outputs by the definition, and the sigma of each."""
    X, Wgu, Wd, dY = (t.double() for t in (X, Wgu, Wd, dY))
    F = Wd.shape[0]
    GU = X @ Wgu
    G, Up = GU[:, :F], GU[:, F:]
    a, slope = _act(G, act)
    H = a * Up
    Y = H @ Wd
    dH = dY @ Wd.T
    dG, dU = dH * Up * slope, dH * a
    dGU = torch.cat((dG, dU), 1)
    # deviations in units of that of one rounding, U / sqrt(3)
    summed = lambda A, B: (2.0 ** -24 / U * 3 ** 0.5) * torch.sqrt((A ** 2) @ (B ** 2) * (A.shape[1] / 6))
    eGU, eH = summed(X, Wgu), summed(dY, Wd.T)
    eG, eU = eGU[:, :F], eGU[:, F:]
    kept = eG ** 2 + (G * 2.0 ** -15 / U) ** 2
    var = dGU ** 2 + torch.cat(((dH * Up * _bend(G, act)) ** 2 * kept + (dH * slope * eU) ** 2 + (Up * slope * eH) ** 2,
                                (dH * slope) ** 2 * kept + (a * eH) ** 2), 1)
    varH = H ** 2 + (Up * slope * eG) ** 2 + (a * eU) ** 2
    sig = lambda prod, out: U / 3 ** 0.5 * torch.sqrt(prod + out ** 2)
    dX, dWgu, dWd = dGU @ Wgu.T, X.T @ dGU, H.T @ dY
    return {"Y": (Y, sig(varH @ Wd ** 2, Y)), "dX": (dX, sig(var @ (Wgu ** 2).T, dX)), "dWgu": (dWgu, sig((X ** 2).T @ var, dWgu)),
            "dWd": (dWd, sig(varH.T @ dY ** 2, dWd))}


def check(got, ref, what):
    out, sigma = ref
    err = (got.double() - out).abs()
    assert bool((err <= 7 * sigma + 1e-30).all()), (what, float((err / (sigma + 1e-30)).max()))
    assert float(err.norm()) <= 1.1 * float(sigma.norm()) + 1e-30, (what, float(err.norm() / sigma.norm()))


# sizes from one token on, over the tiles and the splits of each product
SIZES = [(1, 64, 64), (2, 64, 128), (63, 128, 192), (65, 192, 448), (129, 320, 704), (257, 64, 1024), (1, 576, 256), (1609, 640, 640), (5521, 384, 448), (1772, 2432, 384),
         (831, 384, 5312), (5989, 1344, 2560), (1, 2048, 5440), (40, 2048, 4160), (16, 1088, 2944), (129, 1984, 5440), (70, 64, 8192)]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T,D,F", SIZES)
def test_gated_and_its_gradient(T, D, F, act):
    X, Wgu, Wd, dY = _inputs(T, D, F, seed=T + D + F)
    ctx = block.GatedContext(T + 3, D, F, act=act, training=True)
    Y = ctx.fwd(X, Wgu, Wd)
    dX, dWgu, dWd = ctx.bwd(dY, X, Wgu, Wd)
    ref = reference(X, Wgu, Wd, dY, act)
    for name, got in (("Y", Y), ("dX", dX), ("dWgu", dWgu), ("dWd", dWd)):
        check(got, ref[name], name)
    again = ctx.bwd(dY, X, Wgu, Wd)
    assert all(torch.equal(a, b) for a, b in zip(again, (dX, dWgu, dWd)))
    ctx.close()


# few tokens on a serving context: strips of 64 and 128 channels, one to 16 parts of a reduction, one to four groups of 16 tokens
@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("D,F", [(64, 64), (192, 448), (1088, 2944), (320, 8192), (2048, 5440), (4096, 1024)])
@pytest.mark.parametrize("T", [1, 3, 16, 17, 33, 64])
def test_serving_few_tokens(T, D, F, act):
    X, Wgu, Wd, dY = _inputs(T, D, F, seed=T + D + F)
    ctx = block.GatedContext(64, D, F, act=act)
    Y = ctx.fwd(X, Wgu, Wd)
    check(Y, reference(X, Wgu, Wd, dY, act)["Y"], "Y")
    assert torch.equal(ctx.fwd(X, Wgu, Wd), Y)
    X2 = X.clone()
    X2[T - 1] = float("nan")                     # the last token leaves the others alone
    assert torch.equal(ctx.fwd(X2, Wgu, Wd)[:T - 1], Y[:T - 1])
    ctx.close()


@pytest.mark.gpu
def test_gradient_by_differences():
    """The gradient of sum(Y dY) along a direction of every input, by central differences of the definition."""
    T, D, F = 40, 64, 128
    X, Wgu, Wd, dY = _inputs(T, D, F, seed=7)
    ctx = block.GatedContext(T, D, F, act="gelu", training=True)
    ctx.fwd(X, Wgu, Wd)
    grads = ctx.bwd(dY, X, Wgu, Wd)
    f = lambda x, wgu, wd: float(((lambda gu: _act(gu[:, :F], "gelu")[0] * gu[:, F:])(x @ wgu) @ wd * dY.double()).sum())
    base = [t.double() for t in (X, Wgu, Wd)]
    g = torch.Generator(device="cuda").manual_seed(1)
    for i, grad in enumerate(grads):
        v = torch.randn(base[i].shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-5
        hi, lo = list(base), list(base)
        hi[i], lo[i] = base[i] + h * v, base[i] - h * v
        want = (f(*hi) - f(*lo)) / (2 * h)
        got = float((grad.double() * v).sum())
        # each element's error is at most 7 sigma, independent of v: the sum's is 7 times the root of the sum of (sigma v)^2
        sigma = reference(X, Wgu, Wd, dY, "gelu")[("dX", "dWgu", "dWd")[i]][1]
        assert abs(got - want) <= 7 * float((sigma * v).norm()) + 1e-6 * abs(want)


@pytest.mark.gpu
def test_tokens_are_apart():
    """NaN and infinity in one token stay in that token's rows of Y and dX, whatever its place in a tile."""
    T, D, F = 70, 192, 320
    X, Wgu, Wd, dY = _inputs(T, D, F, seed=3)
    ctx = block.GatedContext(T, D, F, training=True)
    Y = ctx.fwd(X, Wgu, Wd)
    dX = ctx.bwd(dY, X, Wgu, Wd)[0]
    bad = [0, 33, 69]
    X2 = X.clone()
    X2[0, 191], X2[33], X2[69, 0] = float("nan"), float("inf"), float("nan")
    Y2 = ctx.fwd(X2, Wgu, Wd)
    dX2 = ctx.bwd(dY, X2, Wgu, Wd)[0]
    good = [t for t in range(T) if t not in bad]
    assert torch.equal(Y2[good], Y[good]) and torch.equal(dX2[good], dX[good])
    assert bool(Y2[bad].isnan().all()) and bool(dX2[bad].isnan().all())


@pytest.mark.gpu
def test_extreme_gates_stay_finite():
    """Gates from -3e4 to 3e4: the activation is 0 or the gate itself, its slope 0 or 1, and nothing turns into NaN."""
    T = D = F = 64
    X = torch.eye(64, dtype=torch.bfloat16, device="cuda")
    Wgu = torch.zeros((D, 2 * F), dtype=torch.bfloat16, device="cuda")
    Wgu[:, :F] = torch.linspace(-3e4, 3e4, 64, device="cuda")[:, None].to(torch.bfloat16)
    Wgu[:, F:] = 1
    Wd = torch.eye(64, dtype=torch.bfloat16, device="cuda")
    for act in ("silu", "gelu"):
        ctx = block.GatedContext(T, D, F, act=act, training=True)
        Y = ctx.fwd(X, Wgu, Wd)
        assert torch.equal(Y, Wgu[:, :F].clamp(min=0).abs())
        dX, dWgu, dWd = ctx.bwd(torch.ones_like(X), X, Wgu, Wd)
        assert all(bool(t.isfinite().all()) for t in (dX, dWgu, dWd))
        assert torch.equal(dWgu[:, :F], (Wgu[:, :F] > 0).to(torch.bfloat16))
        ctx.close()


@pytest.mark.gpu
def test_other_stream_fewer_tokens_and_no_tokens():
    """A context serves any token count up to its own; results do not depend on what it did before; no tokens: zero weight gradients."""
    D, F = 128, 256
    X, Wgu, Wd, dY = _inputs(300, D, F, seed=11)
    ctx = block.GatedContext(300, D, F, training=True)
    full = ctx.fwd(X, Wgu, Wd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        part = ctx.fwd(X[:130].contiguous(), Wgu, Wd)
        grads = ctx.bwd(dY[:130].contiguous(), X[:130].contiguous(), Wgu, Wd)
    side.synchronize()
    fresh = block.GatedContext(130, D, F, training=True)
    assert torch.equal(fresh.fwd(X[:130].contiguous(), Wgu, Wd), part)
    assert all(torch.equal(a, b) for a, b in zip(fresh.bwd(dY[:130].contiguous(), X[:130].contiguous(), Wgu, Wd), grads))
    assert torch.equal(ctx.fwd(X, Wgu, Wd), full)
    none = ctx.fwd(X[:0], Wgu, Wd)
    dX, dWgu, dWd = ctx.bwd(dY[:0], X[:0], Wgu, Wd)
    assert none.shape == (0, D) and dX.shape == (0, D) and not dWgu.any() and not dWd.any()


@pytest.mark.gpu
def test_replayed_in_a_graph():
    T, D, F = 33, 128, 320
    X, Wgu, Wd, dY = _inputs(T, D, F, seed=2)
    ctx = block.GatedContext(T, D, F, training=True)
    run = lambda: (ctx.fwd(X, Wgu, Wd), *ctx.bwd(dY, X, Wgu, Wd))
    run()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        out = run()
    for seed in range(3):
        X.copy_(_inputs(T, D, F, seed=20 + seed)[0])
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.gpu
def test_call_order_and_refusals():
    X, Wgu, Wd, dY = _inputs(8, 64, 64, seed=0)
    ctx = block.GatedContext(8, 64, 64, training=True)
    with pytest.raises(block.Ffn24Error) as e:
        ctx.bwd(dY, X, Wgu, Wd)
    assert e.value.code == -5
    serving = block.GatedContext(8, 64, 64)
    serving.fwd(X, Wgu, Wd)
    with pytest.raises(block.Ffn24Error) as e:
        serving.bwd(dY, X, Wgu, Wd)
    assert e.value.code == -5
    more = torch.cat((X, X))
    with pytest.raises(block.Ffn24Error) as e:
        ctx.fwd(more, Wgu, Wd)
    assert e.value.code == -2
    with pytest.raises(ValueError, match="Wgu: shape"):
        ctx.fwd(X, Wgu[:, :64], Wd)
    with pytest.raises(ValueError, match="contiguous"):
        ctx.fwd(X, Wgu, Wd.T)
    with pytest.raises(ValueError, match="dtype"):
        ctx.fwd(X.float(), Wgu, Wd)
    L, p = block.lib(), lambda t: t.data_ptr()
    assert L.gated_fwd(ctx._h, p(X) + 2, 7, p(Wgu), p(Wd), p(dY), None) == -3 and L.gated_fwd(ctx._h, None, 8, p(Wgu), p(Wd), p(dY), None) == -1
    assert L.gated_fwd(ctx._h, p(X), -1, p(Wgu), p(Wd), p(dY), None) == -2


def test_refusals_without_a_gpu():
    import ctypes
    L, h = block.lib(), ctypes.c_void_p()
    make = lambda T=8, D=64, F=64, gate=0, flags=0: L.gated_ctx_create(ctypes.byref(h), T, D, F, gate, flags)
    assert make(T=0) == -2 and make(T=(1 << 20) + 1) == -2 and make(D=32) == -2 and make(D=96) == -2 and make(F=0) == -2 and make(F=100) == -2
    assert make(D=(1 << 18) + 64) == -2 and make(gate=2) == -4 and make(flags=2) == -5 and L.gated_ctx_create(None, 8, 64, 64, 0, 0) == -1
    assert h.value is None and L.gated_ctx_destroy(None) == 0
    assert L.gated_fwd(None, None, 0, None, None, None, None) == -1 and L.gated_bwd(None, None, None, None, None, None, None, None, None) == -1
    with pytest.raises(ValueError, match="act"):
        block.GatedContext(8, 64, 64, act="relu")
