"""The mixture of experts for few tokens: the choice exactly as the definition in 64 bits has it, shares and results within the bounds of serve_reference."""
import ctypes

import pytest
import torch

import serve_reference as ref
from paper_2503_16672_amd import serve
from paper_2503_16672_amd.ffn24 import Ffn24Error

BF16, F32 = torch.bfloat16, torch.float32
pytestmark = pytest.mark.gpu


def _normal(shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(BF16)


def _weights(D, F, E, seed=2):
    return _normal((D, E), seed, 2 * D ** -0.5), _normal((E, D, 2 * F), seed + 1, D ** -0.5), _normal((E, F, D), seed + 2, F ** -0.5)


def _run(ctx, X):
    picks, shares = torch.full((X.shape[0], ctx.k), -1, dtype=torch.int32, device="cuda"), torch.empty((X.shape[0], ctx.k), dtype=F32, device="cuda")
    return ctx.fwd(X, experts=picks, shares=shares), picks, shares


def _check(ctx, X, Wr, Wgu, Wd, act, renormalise, weights):
    Y, picks, shares = _run(ctx, X)
    want, p, dp = ref.route(X, Wr, ctx.k, renormalise)
    assert torch.equal(picks.long(), want)
    assert bool(((shares.double() - p).abs() <= dp).all()), float(((shares.double() - p).abs() / dp).max())
    y, d = ref.moe(X, Wr, Wgu, Wd, ctx.k, act, renormalise, weights == "mx4")
    assert ref.holds(Y, y, d), float(((Y.double() - y).abs() / (d + ref.U * y.abs())).max())
    return Y


CASES = [(1, 64, 64, 1, 1), (1, 2048, 1024, 32, 4), (2, 128, 192, 5, 2), (7, 320, 704, 24, 3), (8, 1024, 512, 64, 8), (16, 192, 320, 8, 8), (17, 576, 128, 100, 7), (33, 64, 448, 17, 5),
         (64, 512, 320, 256, 16), (64, 256, 192, 3, 1), (40, 4096, 64, 16, 2), (5, 64, 4160, 7, 3), (48, 128, 128, 128, 16), (1, 128, 8256, 4, 2), (64, 4416, 192, 5, 4),
         (64, 16384, 64, 256, 16), (1, 16384, 128, 256, 16), (50, 64, 65536, 4, 3), (1, 64, 65536, 3, 3), (64, 1536, 512, 16, 16)]


@pytest.mark.parametrize("weights", ["bf16", "mx4"])
@pytest.mark.parametrize("T,D,F,E,k", CASES)
def test_layer(T, D, F, E, k, weights):
    act, renormalise = ("silu", "gelu")[T % 2], bool((T + k) % 3)
    X, (Wr, Wgu, Wd) = _normal((T, D), 1), _weights(D, F, E)
    ctx = serve.MoeContext(min(T + 3, 64), Wr, Wgu, Wd, k, act=act, renormalise=renormalise, weights=weights)
    Y = _check(ctx, X, Wr, Wgu, Wd, act, renormalise, weights)
    assert torch.equal(ctx.fwd(X), Y)                             # (results repeat, with or without the choice given out)
    _check(ctx, X[:(T + 1) // 2].contiguous(), Wr, Wgu, Wd, act, renormalise, weights)
    other = _weights(D, F, E, seed=12)
    ctx.set_weights(*other)
    _check(ctx, X, *other, act, renormalise, weights)
    ctx.close()


@pytest.mark.parametrize("weights", ["bf16", "mx4"])
@pytest.mark.parametrize("T", [5, 20, 64])
def test_every_token_chooses_the_same_experts(T, weights):
    """One expert has all tokens, the others none."""
    D, F, E, k = 128, 192, 40, 3
    X, (Wr, Wgu, Wd) = _normal((T, D), 1), _weights(D, F, E)
    X[:, 0] = 8
    Wr[0] = -8
    Wr[0, [3, 17, 39]] = torch.tensor([8.0, 16.0, 24.0], dtype=BF16, device="cuda")
    ctx = serve.MoeContext(T, Wr, Wgu, Wd, k, weights=weights)
    _check(ctx, X, Wr, Wgu, Wd, "silu", True, weights)
    assert _run(ctx, X)[1].tolist() == [[39, 17, 3]] * T


def test_equal_and_near_logits():
    """Among equals the lowest index; two logits that fp32 sums could not tell apart are told apart."""
    T, D, F, E, k = 12, 1024, 64, 30, 6
    X, (Wr, Wgu, Wd) = _normal((T, D), 1), _weights(D, F, E)
    Wr[:, 10:20] = Wr[:, :10]
    Wr[:, 20:] = Wr[:, :10]
    X[:, 0] = 2.0 ** -20
    Wr[0] = 0
    Wr[0, 20:] = 2.0 ** -10                                       # (2^-30 beside a sum of about 1)
    for renormalise in (True, False):
        ctx = serve.MoeContext(T, Wr, Wgu, Wd, k, renormalise=renormalise)
        _check(ctx, X, Wr, Wgu, Wd, "silu", renormalise, "bf16")
        picks = _run(ctx, X)[1]
        assert bool((picks[:, 0] >= 20).all()) and bool((picks[:, 1] < 10).all()) and bool((picks[:, 2] == picks[:, 1] + 10).all())


@pytest.mark.parametrize("weights", ["bf16", "mx4"])
@pytest.mark.parametrize("T", [6, 40])
def test_tokens_are_apart(T, weights):
    """A token with a NaN or an infinity gets experts that exist and a result of NaN; the others get theirs."""
    D, F, E, k = 192, 320, 11, 4
    X, (Wr, Wgu, Wd) = _normal((T, D), 1), _weights(D, F, E)
    ctx = serve.MoeContext(T, Wr, Wgu, Wd, k, weights=weights)
    Y, picks, _ = _run(ctx, X)
    X2 = X.clone()
    X2[1, 5], X2[4, D - 1] = float("nan"), float("inf")
    Y2, picks2, shares2 = _run(ctx, X2)
    rows = [t for t in range(T) if t not in (1, 4)]
    y, d = ref.moe(X, Wr, Wgu, Wd, k, "silu", True, weights == "mx4")
    assert torch.equal(picks2[rows], picks[rows]) and ref.holds(Y2[rows], y[rows], d[rows])
    assert picks2[1].tolist() == [0, 1, 2, 3] and bool(shares2[1].isnan().all())
    assert bool(((picks2 >= 0) & (picks2 < E)).all()) and all(len(set(p)) == k for p in picks2.tolist())
    assert not bool(Y2[[1, 4]].isfinite().any())
    assert torch.equal(ctx.fwd(X), Y)                             # (nothing of it is left in the context)


def test_streams_graphs_and_no_tokens():
    T, D, F, E, k = 9, 256, 192, 20, 3
    X, (Wr, Wgu, Wd) = _normal((T, D), 1), _weights(D, F, E)
    both = [serve.MoeContext(T, Wr, Wgu, Wd, k, weights=w) for w in ("bf16", "mx4")]
    outs, again = [torch.empty_like(X) for _ in both], [torch.empty_like(X) for _ in both]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for c, y in zip(both, again):
            c.fwd(X, Y=y)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for c, y in zip(both, again):
            c.fwd(X, Y=y)
    for i in range(4):
        X.copy_(_normal((T, D), 20 + i))                          # (other experts each time)
        for c, y in zip(both, outs):
            c.fwd(X, Y=y)
        for y in again:
            y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, again))
        y, d = ref.moe(X, Wr, Wgu, Wd, k, "silu", True, False)
        assert ref.holds(outs[0], y, d)
    assert both[0].fwd(X[:0]).shape == (0, D)


def test_refusals():
    D, F, E = 64, 64, 4
    X, (Wr, Wgu, Wd) = _normal((4, D), 1), _weights(D, F, E)
    ctx = serve.MoeContext(4, Wr, Wgu, Wd, 2)
    picks, shares = torch.empty((4, 2), dtype=torch.int32, device="cuda"), torch.empty((4, 2), dtype=F32, device="cuda")
    for call in (lambda: ctx.fwd(X.float()), lambda: ctx.fwd(X[:, :32].contiguous()), lambda: ctx.fwd(X, experts=picks.long(), shares=shares), lambda: ctx.fwd(X, experts=picks[:3], shares=shares),
                 lambda: serve.MoeContext(4, Wr, Wgu, Wd, 2, weights="int8"), lambda: serve.MoeContext(4, Wr, Wgu, Wd, 2, act="relu"), lambda: serve.MoeContext(4, Wr[:, :3], Wgu, Wd, 2),
                 lambda: serve.MoeContext(4, Wr.float(), Wgu, Wd, 2), lambda: serve.MoeContext(4, Wr, Wgu[:, :, :64], Wd, 2)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ctx.fwd(_normal((5, D), 1)), lambda: ctx.fwd(X, experts=picks), lambda: ctx.fwd(X, shares=shares), lambda: serve.MoeContext(65, Wr, Wgu, Wd, 2),
                 lambda: serve.MoeContext(4, Wr, Wgu, Wd, 5), lambda: serve.MoeContext(4, Wr, Wgu, Wd, 0), lambda: serve.MoeContext(4, *_weights(64, 96, 2), 1),
                 lambda: serve.MoeContext(4, *_weights(64, 64, 257), 2), lambda: serve.MoeContext(4, *_weights(64, 64, 32), 17)):
        with pytest.raises(Ffn24Error):
            call()
    h = ctypes.c_void_p()
    L = serve.lib()
    assert L.moe_ctx_create(ctypes.byref(h), 4, D, F, E, 2, 0, 1, 0) == 0
    assert L.moe_fwd(h, X.data_ptr(), 4, torch.empty_like(X).data_ptr(), None, None, None) == -5    # no weights yet
    assert L.moe_ctx_destroy(h) == 0
