"""What mx4 numbers, the products and blocks on them and the mixture of experts are, in 64 bits, and how far fp32 sums and roundings may be off (no GPU code).

A rounding to bf16 is off by at most U = 2^-8 of the value, an fp32 operation by U32 = 2^-24; a sum of n products of mx4 or bf16 values, each exact in fp32, by n U32 of the sum of
their magnitudes, in any order.  The gate's exponential, in fp32: its argument is rounded twice and scaled by log2 e, so it is off by 3 |p| + 4 units of 2^-23 of the value with the
exponential, the sum, the reciprocal and two products behind it."""
import torch

U, U32 = 2.0 ** -8, 2.0 ** -24
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BORDERS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)              # a tie goes to the even code: up at the odd-numbered ones
ACT = {"silu": (1.0, 0.0), "gelu": (1.5957691216057308, 1.5957691216057308 * 0.044715)}


def mx4(x, dim=-1):
    """(codes 0 .. 15, scale codes, values) of x along dim, in blocks of 32; the codes of a block with an infinity or a NaN are 0, its values NaN."""
    x = x.double().movedim(dim, -1)
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = b.abs().amax(dim=-1, keepdim=True)
    good = torch.isfinite(b).all(dim=-1, keepdim=True)
    _, e = torch.frexp(torch.where(good, top, torch.ones_like(top)))
    scale = torch.where(top > 0, (e - 3 + 127).clamp(min=0), torch.zeros_like(e))
    powers = torch.tensor([2.0 ** (i - 127) for i in range(255)], dtype=torch.float64, device=x.device)
    s = powers[scale.long()]
    v = torch.where(good, b, torch.zeros_like(b)) / s
    m = v.abs()
    code = torch.zeros(m.shape, dtype=torch.int64, device=x.device)
    for i, border in enumerate(BORDERS):
        code += (m >= border) if i % 2 else (m > border)
    values = torch.copysign(torch.tensor(VALUES, dtype=torch.float64, device=x.device)[code], v) * s
    code = code + 8 * torch.signbit(v).long()
    values = torch.where(good, values, torch.full_like(values, float("nan")))
    scale = torch.where(good, scale.long(), torch.full_like(scale.long(), 255))
    return code.reshape(x.shape).movedim(-1, dim), scale[..., 0].movedim(-1, dim), values.reshape(x.shape).movedim(-1, dim)


def values(x, dim=-1):
    return mx4(x, dim)[2]


def unpack(codes):
    """[T, K / 2] bytes -> [T, K] codes"""
    return torch.stack((codes & 15, codes >> 4), dim=-1).reshape(codes.shape[0], -1).long()


def decode(codes, scales):
    """The values of codes [T, K] and scale codes [T, K / 32] in 64 bits"""
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), dtype=torch.float64, device=codes.device)
    powers = torch.tensor([2.0 ** (i - 127) for i in range(255)] + [float("nan")], dtype=torch.float64, device=codes.device)
    return table[codes] * powers[scales.long()].repeat_interleave(32, dim=1)


def product(x, w):
    """x w of values that are exact, and how far its fp32 sum may be off"""
    return x @ w, x.shape[1] * U32 * (x.abs() @ w.abs())


def activation(G, Up, dG, dU, act):
    """h = a(G) U, and how far h may be off if G and U are by dG, dU"""
    c1, c3 = ACT[act]
    p = c1 * G + c3 * G ** 3
    a = G * torch.sigmoid(p)
    h = a * Up
    # |a'| <= 1.13 for both gates
    return h, 1.13 * dG * Up.abs() + (a.abs() + 1.13 * dG) * dU + (3 * p.abs() + 4) * 2 * U32 * h.abs()


def narrowed(h, dh):
    """mx4 values of h along its rows, and how far they may be off if h is by dh: a step where a border (or the next power of two of the block's largest) is within dh"""
    v = values(h)
    lo, hi = values((h.abs() - dh).clamp(min=0) * torch.sign(h)), values((h.abs() + dh) * torch.sign(h))
    b = h.abs().reshape(h.shape[0], -1, 32)
    d = dh.reshape(h.shape[0], -1, 32)
    top_lo, top_hi = (b - d).clamp(min=0).amax(-1, keepdim=True), (b + d).amax(-1, keepdim=True)
    turn = torch.frexp(top_lo)[1] != torch.frexp(top_hi)[1]     # the scale may be either
    off = torch.maximum((lo - v).abs(), (hi - v).abs())
    # of the two scales' values: both within half a step of h, the larger scale's step is at most half the block's largest
    both = (top_hi * 0.5).expand_as(b).reshape(h.shape)
    return v, torch.where(turn.expand_as(b).reshape(h.shape), torch.maximum(off, both), off)


def gated_mx4(X, Wgu, Wd, act, narrow=True):
    """(Y, how far it may be off before it is rounded) from values X, Wgu, Wd that the products take (mx4 or bf16, in 64 bits); narrow: h to mx4, otherwise to bf16"""
    F = Wd.shape[0]
    gu, d = product(X, Wgu)
    h, dh = activation(gu[:, :F], gu[:, F:], d[:, :F], d[:, F:], act)
    if narrow:
        h, dh = narrowed(h, dh)
    else:
        dh = dh + U * (h.abs() + dh)
    y = h @ Wd
    return y, dh @ Wd.abs() + F * U32 * ((h.abs() + dh) @ Wd.abs())


def route(X, Wr, k, renormalise):
    """(experts [T, k], shares [T, k], how far those may be off) in 64 bits"""
    logits = X.double() @ Wr.double()
    key = torch.where(torch.isnan(logits), torch.full_like(logits, -float("inf")), logits)
    nan = torch.isnan(logits)
    T, E = logits.shape
    picks = torch.empty((T, k), dtype=torch.int64, device=X.device)
    left = torch.ones_like(nan)
    for j in range(k):
        best = torch.where(left & ~nan, key, torch.full_like(key, -float("inf")))
        # (the first of the largest; NaN after everything else, infinities below too)
        top = best.amax(dim=1, keepdim=True)
        cand = left & ~nan & (key == top)
        cand = torch.where(cand.any(dim=1, keepdim=True), cand, left)
        picks[:, j] = cand.int().argmax(dim=1)
        left[torch.arange(T, device=X.device), picks[:, j]] = False
    l = logits.gather(1, picks)
    e = torch.exp(l - l[:, :1])
    total = e.sum(1, keepdim=True) if renormalise else torch.exp(logits - l[:, :1]).sum(1, keepdim=True)
    p = e / total
    # the difference, the exponential (2 units), the sum and the division, each of 2^-23 at most, and what the largest difference does to the sum; a share below the
    # normal range of fp32 (2^-126; logits 88 apart) may be 0
    return picks, p, p * ((l - l[:, :1]).abs() + 16 + 8 * E * U32) * 2 * U32 + 2.0 ** -126


def moe(X, Wr, Wgu, Wd, k, act, renormalise, narrow):
    """(Y, how far it may be off before it is rounded) of bf16 tokens and weights"""
    T = X.shape[0]
    picks, p, dp = route(X, Wr, k, renormalise)
    x = values(X) if narrow else X.double()
    Y, dY = torch.zeros_like(x), torch.zeros_like(x)
    for e in range(Wd.shape[0]):
        t, j = torch.nonzero(picks == e, as_tuple=True)
        if t.numel() == 0:
            continue
        y, d = gated_mx4(x[t], *(values(w[e], 0) if narrow else w[e].double() for w in (Wgu, Wd)), act, narrow)
        w, dw = p[t, j, None], dp[t, j, None]
        Y[t] += w * y
        dY[t] += w * d + dw * (y.abs() + d) + (k + 10) * U32 * w * (y.abs() + d)
    return Y, dY


def holds(got, y, d):
    """Whether bf16 `got` is y within d and its rounding"""
    return bool(((got.double() - y).abs() <= d + U * (y.abs() + d) + 1e-38).all())
