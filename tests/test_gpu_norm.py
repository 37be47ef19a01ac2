"""Layer norm, forward and backward, against its definition in 64 bits.

Tolerances follow from the arithmetic: u = 2^-24 of a value is half a unit of its last place in fp32, 2^-8 in bf16 (24 and 8 bits).  A sum over D values in lanes, waves and rows adds
at most ~100 times one after the other, so it is off by 100 u of the sum of magnitudes; what is computed from it inherits that."""
import numpy as np
import pytest
import torch

from paper_2503_16672_amd import block

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


def _case(T, D, dtype, seed, offset=0.5):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)
    x = {"X": (n(T, D) * (0.5 + n(D).abs()) + offset * n(D)).to(dtype), "R": n(T, D).to(dtype), "w": 1 + 0.3 * n(D), "b": 0.3 * n(D),
         "dY": n(T, D).to(dtype), "dS": n(T, D).to(dtype)}
    return x, {k: v.cuda() for k, v in x.items()}


def _ref(S, w, b, eps):
    S, w = S.double(), w.double()
    mean = S.mean(dim=1)
    c = S - mean[:, None]
    rstd = 1 / torch.sqrt((c * c).mean(dim=1) + eps)
    xh = c * rstd[:, None]
    return mean, rstd, xh, xh * w + (0 if b is None else b.double())


def _within(got, ref, tol, what):
    bad = (got.double().cpu() - ref).abs() - tol
    assert bool((bad <= 0).all()), (what, float(bad.max()), tuple(ref.shape))


def _check(x, d, dtype, residual, bias, grad_s, eps=1e-5):
    T, D = x["X"].shape
    b = x["b"] if bias else None
    Y, S, mean, rstd = block.layer_norm_fwd(d["X"], d["w"], d["b"] if bias else None, eps, residual=d["R"] if residual else None)
    want = (x["X"].float() + x["R"].float()).to(dtype) if residual else x["X"]
    assert torch.equal(S.cpu(), want)
    rmean, rrstd, xh, ry = _ref(want, x["w"], b, eps)
    w, s = x["w"].double(), want.double()
    size = s.abs().mean(dim=1)                                        # of the mean's summands
    _within(mean, rmean, 100 * U * size + U * rmean.abs(), "mean")
    loose = rrstd * size * 100 * U                                    # of a centred, scaled value
    _within(rstd, rrstd, rrstd * (100 * U + loose), "rstd")
    dxh = loose[:, None] * (1 + xh.abs()) + 110 * U * xh.abs()
    _within(Y, ry, HALF[dtype] * 1.01 * ry.abs() + dxh * w.abs() + 4 * U * (xh * w).abs() + 2 * U * ry.abs(), "Y")

    dX, dw, db = block.layer_norm_bwd(d["dY"], S, d["w"], mean, rstd, dS=d["dS"] if grad_s else None)
    dy, ds = x["dY"].double(), x["dS"].double() if grad_s else torch.zeros_like(s)
    p = dy * w
    m1, m2 = p.mean(dim=1, keepdim=True), (p * xh).mean(dim=1, keepdim=True)
    rdx = rrstd[:, None] * (p - m1 - xh * m2) + ds
    a1, a2 = p.abs().mean(dim=1, keepdim=True), (p * xh).abs().mean(dim=1, keepdim=True)
    off = 110 * U * (p.abs() + a1 + xh.abs() * a2) + dxh * a2 + xh.abs() * (p.abs() * dxh).mean(dim=1, keepdim=True)
    off = off + (loose[:, None] + 100 * U) * (p - m1 - xh * m2).abs()
    _within(dX, rdx, HALF[dtype] * 1.01 * rdx.abs() + rrstd[:, None] * off + 4 * U * ds.abs(), "dX")
    _within(dw, (dy * xh).sum(dim=0), 200 * U * (dy * xh).abs().sum(dim=0) + (dy.abs() * dxh).sum(dim=0), "dw")
    _within(db, dy.sum(dim=0), 200 * U * dy.abs().sum(dim=0), "db")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,D", [(1, 1), (3, 7), (5, 8), (1, 4096), (2, 512), (4, 513), (1031, 1001), (1025, 520), (1024, 1024), (37, 2048), (1200, 2056),
                                 (1030, 4096), (9, 5000), (7, 8192), (3, 9001), (600, 8200), (2, 16384)])
def test_norm_and_its_gradient(T, D, dtype):
    x, d = _case(T, D, dtype, seed=T + D)
    _check(x, d, dtype, residual=True, bias=True, grad_s=True)
    _check(x, d, dtype, residual=False, bias=False, grad_s=False)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_offset_keeps_the_variance(dtype):
    """Values around 1000 with a spread of a few: the variance must come from centred values (squares of fp32 would leave nothing of it)."""
    x, d = _case(6, 4096, dtype, seed=3)
    x["X"] = (x["X"].float() * 4 + 1000).to(dtype)
    d["X"] = x["X"].cuda()
    _check(x, d, dtype, residual=False, bias=True, grad_s=True)


@pytest.mark.gpu
def test_gradient_by_differences():
    x, d = _case(3, 40, torch.float32, seed=5)
    f = lambda s: float((_ref(s, x["w"], x["b"], 1e-5)[3] * x["dY"].double()).sum())
    Y, S, mean, rstd = block.layer_norm_fwd(d["X"], d["w"], d["b"])
    dX = block.layer_norm_bwd(d["dY"], S, d["w"], mean, rstd)[0].cpu()
    h = 1e-5
    for t, i in [(0, 0), (1, 17), (2, 39)]:
        hi, lo = x["X"].double(), x["X"].double()
        hi[t, i] += h
        lo[t, i] -= h
        assert abs((f(hi) - f(lo)) / (2 * h) - float(dX[t, i])) <= 1e-4 * (1 + abs(float(dX[t, i])))


@pytest.mark.gpu
def test_rows_are_apart_and_constant_rows_are_finite():
    """A row of NaN or infinity stays in its row of every per-token output; a constant row is its bias."""
    x, d = _case(6, 1000, torch.bfloat16, seed=1)
    clean = block.layer_norm_fwd(d["X"], d["w"], d["b"])
    dirty = d["X"].clone()
    dirty[1, 5], dirty[4] = float("nan"), float("inf")
    dirty[2] = 3.0
    got = block.layer_norm_fwd(dirty, d["w"], d["b"])
    for t in (0, 3, 5):
        assert torch.equal(got[0][t], clean[0][t]) and got[2][t] == clean[2][t]
    assert bool(got[0][1].isnan().all()) and bool(got[0][4].isnan().all())
    assert torch.equal(got[0][2], d["b"].to(torch.bfloat16))
    g, h = block.layer_norm_bwd(d["dY"], dirty, d["w"], got[2], got[3])[0], block.layer_norm_bwd(d["dY"], d["X"], d["w"], clean[2], clean[3])[0]
    for t in (0, 3, 5):
        assert torch.equal(g[t], h[t])


@pytest.mark.gpu
def test_in_place_other_stream_and_repeated():
    """S in X's place, Y in R's; on a stream of its own; the sums over tokens repeat bit for bit."""
    x, d = _case(1500, 1024, torch.bfloat16, seed=8)
    Y, S, mean, rstd = block.layer_norm_fwd(d["X"], d["w"], d["b"], residual=d["R"])
    first = block.layer_norm_bwd(d["dY"], S, d["w"], mean, rstd, dS=d["dS"])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        X, dS = d["X"].clone(), d["dS"].clone()
        out = torch.empty_like(X)
        p = lambda t: t.data_ptr()
        s = torch.cuda.current_stream().cuda_stream
        assert block.lib().layer_norm_fwd(p(X), p(d["R"]), p(d["w"]), p(d["b"]), 1500, 1024, 1e-5, 0, p(X), p(out), None, None, s) == 0
        n = block.lib().layer_norm_bwd_scratch(1500, 1024)
        scratch, dw, db = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(1024, device="cuda"), torch.empty(1024, device="cuda")
        assert block.lib().layer_norm_bwd(p(d["dY"]), p(X), p(d["w"]), p(mean), p(rstd), p(dS), 1500, 1024, 0, p(dS), p(dw), p(db), p(scratch), s) == 0
    side.synchronize()
    assert torch.equal(X, S) and torch.equal(out, Y)
    assert torch.equal(dS, first[0]) and torch.equal(dw, first[1]) and torch.equal(db, first[2])


@pytest.mark.gpu
def test_no_tokens():
    w = torch.ones(100, device="cuda")
    X = torch.empty((0, 100), dtype=torch.bfloat16, device="cuda")
    Y, S, mean, rstd = block.layer_norm_fwd(X, w, w)
    assert Y.shape == (0, 100) and mean.shape == (0,)
    dX, dw, db = block.layer_norm_bwd(X, X, w, mean, rstd)
    assert dX.shape == (0, 100) and not dw.any() and not db.any()


@pytest.mark.gpu
def test_replayed_in_a_graph():
    x, d = _case(300, 768, torch.bfloat16, seed=2)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    run = lambda: (lambda f: (*f, *block.layer_norm_bwd(d["dY"], f[1], d["w"], f[2], f[3], dS=d["dS"])))(block.layer_norm_fwd(d["X"], d["w"], d["b"], residual=d["R"]))
    run()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        out = run()
    for seed in range(3):
        d["X"].copy_(_case(300, 768, torch.bfloat16, seed=10 + seed)[1]["X"])
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals_without_a_gpu():
    L = block.lib()
    a = 0x1000
    fwd = lambda X=a, R=None, w=a, b=None, T=4, D=8, eps=1e-5, t=0, S=None, Y=a, m=None, r=None: L.layer_norm_fwd(X, R, w, b, T, D, eps, t, S, Y, m, r, None)
    assert fwd(t=2) == -4 and fwd(T=-1) == -2 and fwd(D=0) == -2 and fwd(D=16385) == -2 and fwd(eps=0.0) == -2 and fwd(eps=float("nan")) == -2
    assert fwd(X=None) == -1 and fwd(w=None) == -1 and fwd(Y=None) == -1 and fwd(R=a) == -1 and fwd(S=a) == -1 and fwd(m=a) == -1
    assert fwd(X=a + 2) == -3 and fwd(Y=a + 8) == -3 and fwd(b=a + 4) == -3
    assert fwd(X=None, T=0) == 0
    bwd = lambda dY=a, S=a, w=a, m=a, r=a, dS=None, T=4, D=8, t=0, dX=a, dw=a, db=None, s=a: L.layer_norm_bwd(dY, S, w, m, r, dS, T, D, t, dX, dw, db, s, None)
    assert bwd(t=-1) == -4 and bwd(T=-1) == -2 and bwd(D=20000) == -2 and bwd(dY=None) == -1 and bwd(dw=None) == -1 and bwd(s=None) == -1 and bwd(m=None) == -1
    assert bwd(dS=a + 2) == -3 and bwd(s=a + 4) == -3
    assert L.layer_norm_bwd_scratch(4, 0) == -1 and L.layer_norm_bwd_scratch(-1, 8) == -1 and L.layer_norm_bwd_scratch(0, 8) == 0
    assert L.layer_norm_bwd_scratch(1, 8) == 64


def test_binding_refuses_what_does_not_fit():
    X, w = torch.zeros((4, 16), dtype=torch.bfloat16), torch.ones(16)
    with pytest.raises(ValueError, match="CUDA"):
        block.layer_norm_fwd(X, w)
    with pytest.raises(ValueError, match="dtype"):
        block.layer_norm_fwd(X.half(), w)
    with pytest.raises(ValueError, match="weight: shape"):
        block.layer_norm_fwd(X, torch.ones(8))
    with pytest.raises(ValueError, match="residual: dtype"):
        block.layer_norm_fwd(X, w, residual=X.float())
