"""The reference of the mx4 and expert tests against the definitions by other ways (no GPU)."""
import itertools
import math

import pytest
import torch

import serve_reference as ref


def _nearest(x, s):
    """By search over all sixteen values: the nearest, of two the one with the even code"""
    best = min(range(8), key=lambda c: (abs(abs(x) / s - ref.VALUES[c]), c % 2))
    return best + (8 if math.copysign(1.0, x) < 0 else 0)


def test_codes_against_a_search():
    xs = [v * 2.0 ** e for v in (0.0, 0.25, 0.5, 0.6, 0.75, 1.0, 1.25, 1.3, 1.5, 1.75, 2.25, 2.5, 3.0, 3.5, 3.9, 4.0, 5.0, 5.5, 6.0, 7.0, 7.9) for e in (-3, 0, 2)]
    for top in (1.0, 4.0, 6.5, 7.99, 8.0, 1e-30, 2.0 ** -126, 1e-40, 3e38):
        row = torch.tensor([top, *[x * top / 32 for x in xs][:31]], dtype=torch.float64)
        row[1::2] *= -1
        code, scale, values = ref.mx4(row[None])
        s = 2.0 ** max(math.floor(math.log2(top)) - 2, -127)
        assert int(scale) == round(math.log2(s)) + 127
        for x, c, v in zip(row.tolist(), code[0].tolist(), values[0].tolist()):
            assert c == _nearest(x, s) and v == (-1 if c & 8 else 1) * ref.VALUES[c & 7] * s
        assert torch.equal(ref.decode(code, scale), values)


def test_blocks_that_are_not_numbers():
    x = torch.ones((2, 64))
    x[0, 3], x[1, 40] = float("nan"), -float("inf")
    code, scale, values = ref.mx4(x)
    assert scale.tolist() == [[255, 125], [125, 255]]
    assert torch.isnan(values).tolist() == [[True] * 32 + [False] * 32, [False] * 32 + [True] * 32]
    assert ref.mx4(torch.zeros((1, 32)))[1].tolist() == [[0]]


@pytest.mark.parametrize("renormalise", [True, False])
def test_route_takes_the_largest_and_the_first_of_equals(renormalise):
    Wr = torch.tensor([[1.0, 3.0, 3.0, 2.0, 3.0, float("nan")]])
    picks, p, _ = ref.route(torch.ones((1, 1)), Wr, 4, renormalise)
    assert picks.tolist() == [[1, 2, 4, 3]]
    if renormalise:
        assert abs(float(p.sum()) - 1) < 1e-12
    X = torch.randn((40, 8), generator=torch.Generator().manual_seed(0))
    Wr = torch.randn((8, 12), generator=torch.Generator().manual_seed(1))
    picks, p, _ = ref.route(X, Wr, 3, renormalise)
    l = X.double() @ Wr.double()
    assert torch.equal(picks, torch.topk(l, 3, dim=1).indices)
    want = torch.softmax(l, 1).gather(1, picks)
    assert torch.allclose(p, want / want.sum(1, keepdim=True) if renormalise else want, atol=1e-14)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_bounds_hold_in_fp32(act):
    """The same in fp32, one operation after the other, stays within the bounds."""
    g = torch.Generator().manual_seed(5)
    X, Wgu, Wd = (torch.randn(s, generator=g) for s in ((30, 256), (256, 384), (192, 64)))
    x, wgu, wd = ref.values(X), ref.values(Wgu / 16, 0), ref.values(Wd / 14, 0)
    y, d = ref.gated_mx4(x, wgu, wd, act)
    gu = x.float() @ wgu.float()
    c1, c3 = ref.ACT[act]
    G, Up = gu[:, :192], gu[:, 192:]
    h = G * (1 / (1 + torch.exp(-(c1 * G + c3 * G * G * G)))) * Up
    assert bool(((ref.values(h).float() @ wd.float()).double() - y).abs().le(d).all())
    # and they are tight enough to show a fault: a token none of whose values is near a border has the sums' bound alone, (256 + 192) 2^-24 of sums of magnitudes
    assert float(d.median()) < 1e-3 * float(y.abs().mean())


def test_a_step_of_the_scale_is_allowed_where_it_may_turn():
    h = torch.full((1, 32), 0.3, dtype=torch.float64)
    h[0, 0] = 4.0
    v, off = ref.narrowed(h, torch.full_like(h, 1e-9))
    other = ref.values(h - 1e-9 * torch.sign(h))
    assert bool(((other - v).abs() <= off).all()) and not torch.equal(other, v)
