"""Norm, gated block and experts one behind the other as they are served, every sublayer held to its definition on the stream it was given; and tensors beyond 4 GiB."""
import pytest
import torch

import serve_reference as ref
from paper_2503_16672_amd import serve
from paper_2503_16672_amd.sublayer import ExpertSublayer, GatedSublayer

BF16, F32 = torch.bfloat16, torch.float32
pytestmark = pytest.mark.gpu


def _normal(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(BF16)


def _norm(s):
    """The norm of the stored sum in bf16: it is tested against 64 bits elsewhere, so the products behind it are held to what it gives here."""
    from paper_2503_16672_amd import block
    return block.layer_norm_fwd(s, torch.ones(s.shape[1], device="cuda"), torch.zeros(s.shape[1], device="cuda"))[0]


@pytest.mark.parametrize("T", [1, 7, 16, 33, 64])
def test_a_stack_of_sublayers(T):
    D, F, E, k = 512, 1408, 12, 3
    x, stream = _normal((T, D), 1), _normal((T, D), 2)
    first, second, third = GatedSublayer(T, D, F, seed=3), ExpertSublayer(T, D, 704, E, k, seed=4, weights="mx4"), ExpertSublayer(T, D, 704, E, k, act="gelu", seed=5)
    mx4 = first.quantised("mx4")
    a, s = first.serve(x, stream, mx4)
    assert torch.equal(s, (x.float() + stream.float()).to(BF16))
    y, d = ref.gated_mx4(ref.values(_norm(s)), ref.values(first.Wgu, 0), ref.values(first.Wd, 0), "silu")
    assert ref.holds(a, y, d)
    b, u = second.serve(a, s)
    assert torch.equal(u, (a.float() + s.float()).to(BF16))
    y, d = ref.moe(_norm(u), second.Wr, second.Wgu, second.Wd, k, "silu", True, True)
    assert ref.holds(b, y, d)
    c, v = third.serve(b, u)
    y, d = ref.moe(_norm(v), third.Wr, third.Wgu, third.Wd, k, "gelu", True, False)
    assert ref.holds(c, y, d)
    with pytest.raises(ValueError):
        first.quantised("int4")


def test_two_streams_at_once():
    """Contexts of their own, one set of weights and tokens: calls that run beside each other give what they give alone, with other sizes before and after."""
    D, F, E, k = 512, 704, 12, 3
    Wr, Wgu, Wd = _normal((D, E), 1), _normal((E, D, 2 * F), 2) * D ** -0.5, _normal((E, F, D), 3) * F ** -0.5
    X, W4 = _normal((64, D), 4), serve.Mx4Weight(Wgu[0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    sets = [(serve.MoeContext(64, Wr, Wgu, Wd, k, weights=w), serve.GatedMx4Context(64, Wgu[i].contiguous(), Wd[i].contiguous())) for i, w in enumerate(("bf16", "mx4"))]
    work = lambda c, t: (c[0].fwd(X[:t]), c[1].fwd(X[:t]), serve.linear_mx4(X[:t], W4))
    sizes = (64, 1, 17, 5, 64, 33)
    want = [[work(c, t) for t in sizes] for c in sets]
    torch.cuda.synchronize()
    got = [[] for _ in sets]
    for _ in range(20):
        for c, s, out in zip(sets, streams, got):
            with torch.cuda.stream(s):
                out[:] = [work(c, t) for t in sizes]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for one, other in zip(want, got) for x, y in zip(one, other) for a, b in zip(x, y))


def _large(shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(shape, dtype=BF16, device="cuda")
    for rows in out.split(max(1, (1 << 28) // shape[1])):
        rows.copy_(torch.randn(rows.shape, generator=g, device="cuda") * scale)
    return out


def test_rounding_beyond_4_gib():
    T, K = 540001, 8192                                          # (8.8 GB in bf16; codes 2.2)
    X = _large((T, K), 1)
    codes, scales = serve.quantise_mx4(X)
    Y = serve.dequantise_mx4(codes, scales)
    for i in (0, 262143, 262144, T - 1000):
        part = slice(i, min(i + 1000, T))
        c, s, v = ref.mx4(X[part])
        assert torch.equal(ref.unpack(codes[part]), c) and torch.equal(scales[part].long(), s) and torch.equal(Y[part].double(), v)


def test_tokens_beyond_4_gib():
    T, K, N = 560001, 16384, 72                                  # (tokens as mx4: 4.9 GB)
    X, W = _large((T, K), 1), _large((K, N), 2, K ** -0.5)
    Y = serve.linear_mx4(X, serve.Mx4Weight(W))
    w = ref.values(W, 0)
    for i in (0, 300000, T - 500):
        part = slice(i, min(i + 500, T))
        assert ref.holds(Y[part], *ref.product(ref.values(X[part]), w))


@pytest.mark.parametrize("T", [3, 70])
def test_weights_beyond_4_gib(T):
    K, N = 16384, 560008                                         # (4.9 GB as mx4)
    X, W = _large((T, K), 1), _large((K, N), 2, K ** -0.5)
    Y = serve.linear_mx4(X, serve.Mx4Weight(W))
    x = ref.values(X)
    for i in (0, 280000, N - 504):
        part = slice(i, min(i + 504, N))
        assert ref.holds(Y[:, part], *ref.product(x, ref.values(W[:, part].contiguous(), 0)))


def test_results_beyond_4_gib():
    T, K, N = 70001, 64, 33000                                   # (Y: 4.6 GB)
    X, W = _large((T, K), 1), _large((K, N), 2, K ** -0.5)
    Y = serve.linear_mx4(X, serve.Mx4Weight(W))
    w = ref.values(W, 0)
    for i in (0, 32000, T - 300):
        part = slice(i, min(i + 300, T))
        assert ref.holds(Y[part], *ref.product(ref.values(X[part]), w))


def test_activations_beyond_4_gib():
    T, D, F = 560001, 64, 16384                                  # (H as mx4: 4.9 GB)
    X, Wgu, Wd = _large((T, D), 1), _large((D, 2 * F), 2, D ** -0.5), _large((F, D), 3, F ** -0.5)
    Y = serve.GatedMx4Context(T, Wgu, Wd).fwd(X)
    wgu, wd = ref.values(Wgu, 0), ref.values(Wd, 0)
    for i in (0, 300000, T - 300):
        part = slice(i, min(i + 300, T))
        assert ref.holds(Y[part], *ref.gated_mx4(ref.values(X[part]), wgu, wd, "silu"))


@pytest.mark.parametrize("weights", ["bf16", "mx4"])
def test_experts_beyond_4_gib(weights):
    T, D, F, E, k = 5, 4096, 4096, 64 if weights == "bf16" else 200, 3      # (6.4 GB in bf16; 200 of them 5.3 GB in mx4)
    X, Wr = _normal((T, D), 1), _normal((D, E), 2) * 2 * D ** -0.5
    Wgu, Wd = _large((E * D, 2 * F), 3, D ** -0.5).view(E, D, 2 * F), _large((E * F, D), 4, F ** -0.5).view(E, F, D)
    X[0] = 0
    X[0, 0] = 1
    Wr[0] = -1
    Wr[0, E - 1] = 4                                             # (one token chooses the last expert)
    ctx = serve.MoeContext(T, Wr, Wgu, Wd, k, weights=weights)
    picks, shares = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), dtype=F32, device="cuda")
    Y = ctx.fwd(X, experts=picks, shares=shares)
    assert int(picks[0, 0]) == E - 1
    y, d = ref.moe(X, Wr, Wgu, Wd, k, "silu", True, weights == "mx4")
    assert ref.holds(Y, y, d)
