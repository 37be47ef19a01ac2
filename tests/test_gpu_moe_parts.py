"""The bf16 experts' activations between the two products: h is held to 2^-16 of it (as the sum of two bf16), so a result is off by the sums, the gate and Y's own rounding alone.

The bound: h's upper 16 bits leave a rest below 2^(e - 7), e the exponent of h; the rest rounded to bf16 is off by at most half a step of a value below that, 2^(e - 16).  The down
product then has 2 F products, each of two bf16 and exact in fp32.

The size of the error: a result is off by no more than the exact one's distance to its nearest bf16 and twice what it was off before it was rounded (that distance changes by
no more than its argument).  Over many results the latter is 2^-16 of their size for h (errors of either sign) and sqrt(n) 2^-24 for sums of n terms, 2^-15 for the largest n here;
a rounding to bf16 is 2^-9.2 of it on average.  2 (2^-16 + 2^-15) / 2^-9.2 < 2^-4.  One bf16 for h adds 2^-9.2 as well: sqrt(2) of the size, and more than the bound where sums are short."""
import subprocess

import pytest
import torch

import serve_reference as ref
from paper_2503_16672_amd import serve
from test_gpu_moe import _normal, _weights
from test_serve_rules import RULE, paths  # noqa: F401

BF16 = torch.bfloat16
HELD = 2.0 ** -16
# every kernel of bf16 experts (below): one token, whole and half strips; up to 16; more, one pass and several; down with strips of 16, 32 and 64 channels, alone and shared
CASES = [(1, 64, 64, 1, 1), (1, 2048, 1024, 32, 4), (1, 256, 4160, 8, 4), (1, 192, 8256, 4, 2), (2, 128, 192, 5, 2), (8, 1024, 512, 64, 8), (16, 192, 320, 8, 8), (17, 576, 128, 100, 7),
         (33, 64, 448, 17, 5), (64, 512, 320, 256, 16), (64, 256, 192, 3, 1), (37, 1088, 704, 24, 3), (64, 4416, 192, 5, 4), (64, 1536, 512, 16, 16), (3, 4096, 64, 8, 2),
         (16, 1344, 64, 4, 2), (8, 1344, 512, 16, 4), (37, 1536, 512, 16, 4), (4, 2624, 1024, 1, 1), (20, 2624, 1024, 1, 1), (9, 2880, 1472, 16, 2), (64, 2624, 1024, 12, 3), (5, 8320, 1024, 3, 2), (64, 2624, 1024, 6, 6),
         (16, 2624, 1024, 1, 1), (2, 2624, 1024, 9, 8), (12, 1024, 2048, 7, 2), (50, 1152, 2112, 9, 3)]


def _expected(X, Wr, Wgu, Wd, k, act, renormalise, kept=lambda h: h):
    """(Y, how far it may be off before it is rounded); kept: what is left of h between the products"""
    picks, p, dp = ref.route(X, Wr, k, renormalise)
    x, F = X.double(), Wd.shape[1]
    Y, dY = torch.zeros_like(x), torch.zeros_like(x)
    for e in range(Wd.shape[0]):
        t, j = torch.nonzero(picks == e, as_tuple=True)
        if t.numel() == 0:
            continue
        wd = Wd[e].double()
        gu, d = ref.product(x[t], Wgu[e].double())
        h, dh = ref.activation(gu[:, :F], gu[:, F:], d[:, :F], d[:, F:], act)
        dh = dh + HELD * (h.abs() + dh)
        # (the two parts' magnitudes are h's and at most 2^-6 of it together)
        y, d = kept(h) @ wd, dh @ wd.abs() + 2 * F * ref.U32 * (1 + 2.0 ** -6) * ((h.abs() + dh) @ wd.abs())
        w, dw = p[t, j, None], dp[t, j, None]
        Y[t] += w * y
        dY[t] += w * d + dw * (y.abs() + d) + (k + 10) * ref.U32 * w * (y.abs() + d)
    return Y, dY


def _size(Y, y):
    """The size of the error, of an exact result's rounding"""
    return float((Y.double() - y).norm() / (y.to(BF16).double() - y).norm())


@pytest.mark.gpu
@pytest.mark.parametrize("act,renormalise", [("silu", True), ("gelu", False)])
@pytest.mark.parametrize("T,D,F,E,k", CASES)
def test_results_are_off_by_no_rounding_of_the_activations(T, D, F, E, k, act, renormalise):
    X, (Wr, Wgu, Wd) = _normal((T, D), T + D), _weights(D, F, E)
    ctx = serve.MoeContext(T, Wr, Wgu, Wd, k, act=act, renormalise=renormalise)
    y, d = _expected(X, Wr, Wgu, Wd, k, act, renormalise)
    Y = ctx.fwd(X)
    assert ref.holds(Y, y, d), float(((Y.double() - y).abs() / (d + ref.U * y.abs())).max())
    assert _size(Y, y) < 1 + 2.0 ** -4, _size(Y, y)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 5, 30])
def test_the_largest_activations(T):
    """A finite h beyond the largest bf16 stays finite; an infinite one gives an infinity, not the NaN of its rest.  The first feature is the tokens' first value: G = 181 / 128 2^63."""
    D = F = 64
    X, Wr, Wgu, Wd = (torch.zeros(s, dtype=BF16, device="cuda") for s in ((T, D), (D, 2), (2, D, 2 * F), (2, F, D)))
    X[:, 0] = 1
    Wr[0, 0] = 1                                                  # (expert 0's share is e / (e + 1))
    Wgu[:, 0, 0] = 181 / 128 * 2.0 ** 63
    Wd[:, 0] = 2.0 ** -100
    Wd[:, 0, 1] = -2.0 ** -100
    ctx = serve.MoeContext(T, Wr, Wgu, Wd, 1)
    for up, want in ((181 / 128 * 2.0 ** 64, 181 * 181 / 2.0 ** 14 * 2.0 ** 27), (2.0 ** 65, float("inf"))):
        Wgu[:, 0, F] = up                                        # (h = 1.9996 2^127; or beyond 2^128)
        ctx.set_weights(Wr, Wgu, Wd)
        Y = ctx.fwd(X).double()
        assert bool((Y[:, 1] == -Y[:, 0]).all()) and bool((Y[:, 2:] == Y[:, :1]).all())
        assert bool(((Y[:, 0] - want).abs() <= ref.U * want).all()) if want < 1e300 else bool((Y[:, 0] == want).all())


@pytest.mark.parametrize("D,F", [(64, 64), (256, 192), (320, 704)])
def test_the_bound_tells_one_bf16_from_two(D, F):
    """The mistake planted in 64 bits: h rounded to one bf16 is told by the error's size, and where sums are short by single results; the sum of two passes both."""
    g = torch.Generator().manual_seed(D)
    X, Wr, Wgu, Wd = ((torch.randn(s, generator=g) * a).to(BF16) for s, a in (((40, D), 1), ((D, 6), 2 * D ** -0.5), ((6, D, 2 * F), D ** -0.5), ((6, F, D), F ** -0.5)))

    def upper(h):
        return (h.float().view(torch.int32) & -65536).view(torch.float32).double()
    y, d = _expected(X, Wr, Wgu, Wd, 2, "silu", True)
    one = _expected(X, Wr, Wgu, Wd, 2, "silu", True, kept=lambda h: h.to(BF16).double())[0]
    two = _expected(X, Wr, Wgu, Wd, 2, "silu", True, kept=lambda h: upper(h) + (h - upper(h)).to(BF16).double())[0]
    assert _size(one.to(BF16), y) > 1 + 2.0 ** -4 > _size(two.to(BF16), y)
    assert ref.holds(two.to(BF16), y, d) and bool(((two - y).abs() <= d).all()) and (D > 256 or not ref.holds(one.to(BF16), y, d))


MAIN = """
#include "%s"
#include <cstdio>
int main() {
  int T, D, F, E, k;
  while (std::scanf(" %%d %%d %%d %%d %%d", &T, &D, &F, &E, &k) == 5) {
    const int groups = ffn24::moe_down_groups(T * k, D, F), slots = T * k < E ? T * k : E;
    std::printf("%%d-%%d-%%s ", T <= 16 ? 1 : 4, groups, ffn24::moe_down_splits(D / (16 * groups), slots * ((F / 32 * groups + 7) / 8)) > 1 ? "shared" : "alone");
  }
}
"""


def test_cases_take_every_kernel_of_bf16_experts(paths, tmp_path):         # noqa: F811
    got = {p for p in paths("m", CASES) if p.startswith("bf16")}
    want = {f"bf16-{p}" for p in ("one-whole", "one-half", "few-8", "few-half", "crowded", "passes-8")}
    assert not want - got, want - got
    (tmp_path / "rule.cpp").write_text(MAIN % RULE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-o", str(tmp_path / "rule"), str(tmp_path / "rule.cpp")], check=True)
    got = set(subprocess.run([str(tmp_path / "rule")], input="\n".join(" ".join(map(str, c)) for c in CASES), capture_output=True, text=True, check=True).stdout.split())
    assert got == {f"{n}-{g}-{s}" for n in (1, 4) for g in (1, 2, 4) for s in ("alone", "shared")}, got
