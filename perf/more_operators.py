"""Cases of more operators around the feed-forward block: microscaled 4-bit numbers (mx4) and the mixture of experts for few tokens.

mx4: every 32 neighbours along the reduction share a power of two; an element is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, in 4 bits.

A case is a dict of plain values.  Its `kind` says what a pass runs:

  mx4_round   T rows of K values to 4-bit codes and scales, and back to values
  linear_mx4  a product of bf16 tokens (T x K, quantised on the way) with mx4 weights (K x N)
  gated_mx4   the gated feed-forward block on mx4 weights, its activations quantised in between
  moe         a mixture-of-experts layer: router, the chosen experts' gated blocks (bf16 or mx4 weights), the sum with the router's shares

Tokens ~ N(0, 1); weights ~ N(0, 1 / fan-in), the router's four times that variance.  K is a multiple of 32, N of 8, D and F of 64, as the entry points
require; T is any (at most 64 for moe).
"""
from __future__ import annotations

import math

import torch

own = False

ACT = {"silu": (1.0, 0.0), "gelu": (2.0 * math.sqrt(2.0 / math.pi), 2.0 * math.sqrt(2.0 / math.pi) * 0.044715)}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LARGEST = 6 * 8192 * 4096 * 16384       # flops of the largest listed pass
LARGEST_EXPERTS = 64 * 4096 * 2048      # experts x D x F of the largest listed layer
MX4_BYTES = 17 / 32                     # a value with its part of the scale


# ---------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # a small layer's activations in fp32, looked at through 4 bits
        dict(name="mx4_round_1031_1056", kind="mx4_round", dtype="f32", T=1031, K=1056),
        # the tokens of the benchmark's training step
        dict(name="mx4_round_16384_4096", kind="mx4_round", dtype="bf16", T=16384, K=4096),
        # the smallest product of 4-bit decoding
        dict(name="linear_mx4_1_2048_8192", kind="linear_mx4", T=1, K=2048, N=8192),
        # a ragged batch of prompts through one layer
        dict(name="linear_mx4_333_1088_4168", kind="linear_mx4", T=333, K=1088, N=4168),
        # prompts through one projection at the sizes of a 7B model
        dict(name="linear_mx4_8192_4096_16384", kind="linear_mx4", T=8192, K=4096, N=16384),
        # sixteen sequences decoding together
        dict(name="gated_mx4_16_4096_16384", kind="gated_mx4", act="silu", T=16, D=4096, F=16384),
        # a short prompt and a small model, odd sizes
        dict(name="gated_mx4_1000_1088_2944", kind="gated_mx4", act="gelu", T=1000, D=1088, F=2944),
        # prompts at the sizes of a 7B model
        dict(name="gated_mx4_8192_4096_16384", kind="gated_mx4", act="silu", T=8192, D=4096, F=16384),
        # one sequence's next token through a small mixture: latency
        dict(name="moe_bf16_1_2048_1024", kind="moe", weights="bf16", act="silu", T=1, D=2048, F=1024, E=32, k=4, renormalise=True),
        # a ragged batch, odd sizes, shares of the softmax over all experts
        dict(name="moe_bf16_37_1088_704", kind="moe", weights="bf16", act="gelu", T=37, D=1088, F=704, E=24, k=3, renormalise=False),
        # eight sequences decoding together on 4-bit experts
        dict(name="moe_mx4_8_4096_2048", kind="moe", weights="mx4", act="silu", T=8, D=4096, F=2048, E=64, k=8, renormalise=True),
        # as many sequences as the layer takes: every expert is chosen
        dict(name="moe_bf16_64_4096_2048", kind="moe", weights="bf16", act="silu", T=64, D=4096, F=2048, E=64, k=8, renormalise=True),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _multiple(x, m, lo, hi):
    return int(min(max(round(x / m) * m, lo), hi // m * m))


def draw(rng):
    kind = rng.choice(["mx4_round", "linear_mx4", "linear_mx4", "gated_mx4", "gated_mx4", "moe", "moe", "moe"])
    while True:
        T = int(_log_uniform(rng, 1, 64.99 if kind == "moe" else 16384.99))
        if kind == "mx4_round":
            case = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), T=T, K=_multiple(_log_uniform(rng, 32, 16384), 32, 32, 16384))
            if case["T"] * case["K"] * (2 if case["dtype"] == "bf16" else 4) <= 16384 * 4096 * 2:
                return case
            continue
        if kind == "linear_mx4":
            case = dict(kind=kind, T=T, K=_multiple(_log_uniform(rng, 256, 16384), 32, 256, 16384), N=_multiple(_log_uniform(rng, 256, 16384), 8, 256, 16384))
        elif kind == "gated_mx4":
            D = _multiple(_log_uniform(rng, 256, 8192), 64, 256, 8192)
            case = dict(kind=kind, act=rng.choice(["silu", "gelu"]), T=T, D=D, F=_multiple(D * rng.uniform(2.0, 4.5), 64, 512, 32768))
        else:
            E = int(_log_uniform(rng, 4, 128.99))
            D = _multiple(_log_uniform(rng, 256, 6144), 64, 256, 6144)
            case = dict(kind=kind, weights=rng.choice(["bf16", "mx4"]), act=rng.choice(["silu", "gelu"]), T=T, D=D,
                        F=_multiple(D * rng.uniform(0.3, 2.5), 64, 128, 8192), E=E, k=rng.randint(1, min(E, 8)), renormalise=rng.random() < 0.7)
            if E * D * case["F"] > LARGEST_EXPERTS:
                continue
        if work(case)["flops"] <= LARGEST:
            return case


# ---------------------------------------------------------------------------------------------- inputs
def _normal(g, shape, scale=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=g).mul_(scale).to(dtype)


def _inputs(case, seed):
    """The tensors of a case, made from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, T = case["kind"], case["T"]
    if kind == "mx4_round":
        K = case["K"]
        scale = torch.empty(K, dtype=torch.float32, device="cuda").normal_(generator=g).exp_()      # some features are larger than others
        return {"X": (_normal(g, (T, K), dtype=torch.float32) * scale).to(TYPES[case["dtype"]])}
    if kind == "linear_mx4":
        return {"X": _normal(g, (T, case["K"])), "W": _normal(g, (case["K"], case["N"]), case["K"] ** -0.5)}
    D, F = case["D"], case["F"]
    if kind == "gated_mx4":
        return {"X": _normal(g, (T, D)), "Wgu": _normal(g, (D, 2 * F), D ** -0.5), "Wd": _normal(g, (F, D), F ** -0.5)}
    E = case["E"]
    x = {"X": _normal(g, (T, D)), "Wr": _normal(g, (D, E), 2.0 * D ** -0.5)}
    x["Wgu"] = torch.empty((E, D, 2 * F), dtype=torch.bfloat16, device="cuda")
    x["Wd"] = torch.empty((E, F, D), dtype=torch.bfloat16, device="cuda")
    for e in range(E):
        x["Wgu"][e] = _normal(g, (D, 2 * F), D ** -0.5)
        x["Wd"][e] = _normal(g, (F, D), F ** -0.5)
    return x


def prepare(case, seed):
    st = {"case": case, **_inputs(case, seed)}
    kind, T, X = case["kind"], case["T"], st["X"]
    if own:
        from paper_2503_16672_amd import serve
        if kind == "mx4_round":
            st["codes"] = torch.empty((T, case["K"] // 2), dtype=torch.uint8, device="cuda")
            st["scales"] = torch.empty((T, case["K"] // 32), dtype=torch.uint8, device="cuda")
            st["Y"] = torch.empty_like(X)
        elif kind == "linear_mx4":
            st["W4"] = serve.Mx4Weight(st["W"])
            st["Y"] = torch.empty((T, case["N"]), dtype=torch.bfloat16, device="cuda")
        elif kind == "gated_mx4":
            st["ctx"] = serve.GatedMx4Context(T, st["Wgu"], st["Wd"], act=case["act"])
            st["Y"] = torch.empty_like(X)
        else:
            st["ctx"] = serve.MoeContext(T, st["Wr"], st["Wgu"], st["Wd"], case["k"], act=case["act"], renormalise=case["renormalise"], weights=case["weights"])
            st["Y"] = torch.empty_like(X)
    elif kind == "linear_mx4":
        st["W"] = _mx4(st["W"].float(), 0)
    elif kind == "gated_mx4":
        st["Wgu"], st["Wd"] = _mx4(st["Wgu"].float(), 0), _mx4(st["Wd"].float(), 0)
    elif kind == "moe" and case["weights"] == "mx4":
        for name in ("Wgu", "Wd"):
            for e in range(case["E"]):                       # (bf16 holds these values exactly)
                st[name][e] = _mx4(st[name][e].float(), 0).to(torch.bfloat16)
    return st


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(st):
    from paper_2503_16672_amd import serve
    kind = st["case"]["kind"]
    if kind == "mx4_round":
        codes, scales = serve.quantise_mx4(st["X"], codes=st["codes"], scales=st["scales"])
        return serve.dequantise_mx4(codes, scales, Y=st["Y"])
    if kind == "linear_mx4":
        return serve.linear_mx4(st["X"], st["W4"], Y=st["Y"])
    return st["ctx"].fwd(st["X"], Y=st["Y"])


def _mx4(x, dim):
    """The mx4 values nearest to a float32 matrix; blocks of 32 along `dim`."""
    b = x.unflatten(dim, (-1, 32))
    d = dim + 1
    field = (b.abs().amax(dim=d, keepdim=True).view(torch.int32) >> 23) & 255        # the exponent of the block's largest
    code = (field - 2).clamp(min=0)
    up = ((254 - code) << 23).view(torch.float32)                                     # 1 / scale
    v = b * up
    m = v.abs()
    step = torch.where(m < 2.0, 0.5, torch.where(m < 4.0, 1.0, 2.0))
    q = (torch.round(m / step) * step).clamp(max=6.0)
    y = torch.where(v < 0.0, -q, q) / up
    return torch.where(field == 255, torch.nan, y).flatten(dim, d)


def _act(x, act):
    c1, c3 = ACT[act]
    return x / (1.0 + torch.exp(-(c1 * x + c3 * x * x * x)))


def _gated(X, Wgu, Wd, act, between=lambda h: h):
    gu = X @ Wgu
    F = Wd.shape[0]
    return between(_act(gu[:, :F], act) * gu[:, F:]) @ Wd


def _run_plain(st):
    case = st["case"]
    kind, X = case["kind"], st["X"].float()
    if kind == "mx4_round":
        return _mx4(X, 1).to(TYPES[case["dtype"]])
    along = lambda h: _mx4(h, 1)
    if kind == "linear_mx4":
        return (along(X) @ st["W"]).to(torch.bfloat16)
    if kind == "gated_mx4":
        return _gated(along(X), st["Wgu"], st["Wd"], case["act"], along).to(torch.bfloat16)
    T, E, k = case["T"], case["E"], case["k"]
    logits = X.double() @ st["Wr"].double()                  # (the choice between near ones is not left to 32 bits)
    top, chosen = torch.sort(logits, dim=1, descending=True, stable=True)
    top, chosen = top[:, :k], chosen[:, :k]
    e = torch.exp(top - top[:, :1])
    total = e.sum(dim=1, keepdim=True) if case["renormalise"] else torch.exp(logits - top[:, :1]).sum(dim=1, keepdim=True)
    share = (e / total).float()
    if case["weights"] == "mx4":
        X = along(X)
    else:
        along = lambda h: h
    Y = torch.zeros_like(X)
    if T * k < E:
        for t in range(T):
            for j in range(k):
                at = chosen[t, j:j + 1]
                Wgu, Wd = st["Wgu"].index_select(0, at)[0].float(), st["Wd"].index_select(0, at)[0].float()
                Y[t:t + 1] += share[t, j] * _gated(X[t:t + 1], Wgu, Wd, case["act"], along)
    else:
        for i in range(E):
            p = (share * (chosen == i)).sum(dim=1, keepdim=True)
            Y += p * _gated(X, st["Wgu"][i].float(), st["Wd"][i].float(), case["act"], along)
    return Y.to(torch.bfloat16)


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    kind, T = case["kind"], case["T"]
    if kind == "mx4_round":
        return {"bytes": 2 * (2 if case["dtype"] == "bf16" else 4) * T * case["K"], "flops": 6 * T * case["K"]}
    if kind == "linear_mx4":
        K, N = case["K"], case["N"]
        return {"bytes": int(MX4_BYTES * K * N) + 2 * T * (K + N), "flops": 2 * T * K * N}
    D, F = case["D"], case["F"]
    if kind == "gated_mx4":
        return {"bytes": int(MX4_BYTES * 3 * D * F) + 4 * T * D, "flops": 6 * T * D * F}
    E, k = case["E"], case["k"]
    experts = E * (1.0 - (1.0 - k / E) ** T)                 # how many different ones T tokens choose, on average
    size = 2 if case["weights"] == "bf16" else MX4_BYTES
    return {"bytes": int(experts * size * 3 * D * F) + 2 * D * E + 4 * T * D, "flops": 6 * T * k * D * F + 2 * T * D * E}


# ---------------------------------------------------------------------------------------------- the same in 64 bits
def _nearest(x, dim):
    """As _mx4, in 64 bits and by comparison with the borders between neighbouring values."""
    b = x.double().unflatten(dim, (-1, 32))
    d = dim + 1
    _, e = torch.frexp(b.abs().amax(dim=d, keepdim=True))
    powers = torch.tensor([2.0 ** n for n in range(-127, 128)], dtype=torch.float64, device=x.device)
    s = powers[(e - 3).clamp(min=-127).long() + 127]
    b = b / s
    m = b.abs()
    n = torch.zeros_like(m, dtype=torch.uint8)
    for border, tie_up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        n += (m >= border) if tie_up else (m > border)
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    return (torch.copysign(values[n.long()], b) * s).flatten(dim, d)


def exact(case, seed):
    x = _inputs(case, seed)
    kind = case["kind"]
    if kind == "mx4_round":
        return _nearest(x["X"], 1)
    if kind == "linear_mx4":
        return _nearest(x["X"], 1) @ _nearest(x["W"], 0)
    c1, c3 = ACT[case["act"]]

    def block(X, Wgu, Wd, narrow):
        G, U = (X @ Wgu).chunk(2, dim=1)
        H = torch.sigmoid(c1 * G + c3 * G.pow(3)).mul_(G).mul_(U)
        return (_nearest(H, 1) if narrow else H) @ Wd

    if kind == "gated_mx4":
        return block(_nearest(x["X"], 1), _nearest(x["Wgu"], 0), _nearest(x["Wd"], 0), True)
    narrow = case["weights"] == "mx4"
    logits = x["X"].double() @ x["Wr"].double()
    left = logits.clone()
    rows = torch.arange(case["T"], device=left.device)
    picks = []
    for _ in range(case["k"]):                               # the largest that is left, the first of equals
        best = (left == left.amax(dim=1, keepdim=True)).int().argmax(dim=1)
        picks.append(best)
        left[rows, best] = -math.inf
    picked = torch.zeros_like(logits, dtype=torch.bool)
    for p in picks:
        picked[rows, p] = True
    share = torch.softmax(logits.masked_fill(~picked, -math.inf) if case["renormalise"] else logits, dim=1) * picked
    X = _nearest(x["X"], 1) if narrow else x["X"].double()
    Y = torch.zeros_like(X)
    for e in range(case["E"]):
        at = torch.nonzero(picked[:, e])[:, 0]
        if at.numel():
            Wgu, Wd = (_nearest(w, 0) if narrow else w.double() for w in (x["Wgu"][e], x["Wd"][e]))
            Y[at] += share[at, e, None] * block(X[at], Wgu, Wd, narrow)
    return Y
