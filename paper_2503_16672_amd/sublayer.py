"""The pre-norm gated feed-forward sublayer of a transformer on the operators of `block`: trained in bf16, served in bf16 or int8.

    stream' = stream + x;   x' = FFN(LayerNorm(stream'))

x is what the sublayer before added to the residual stream; the sum is left to the norm of the sublayer after, which reads both anyway.

    python -m paper_2503_16672_amd.sublayer      # trains two sublayers on a synthetic target, then answers single tokens in bf16 and int8
"""
from __future__ import annotations

import torch

from . import block


class GatedSublayer:
    """One sublayer's weights, and its contexts for up to T tokens a call."""

    def __init__(self, T: int, D: int, F: int, act: str = "silu", eps: float = 1e-5, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda shape, scale: (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16)
        self.T, self.act, self.eps = T, act, eps
        self.norm_weight, self.norm_bias = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
        self.Wgu, self.Wd = new((D, 2 * F), D ** -0.5), new((F, D), F ** -0.5)
        self.training = block.GatedContext(T, D, F, act=act, training=True)
        self.serving = block.GatedContext(T, D, F, act=act)

    def forward(self, x, stream):
        """(x', stream'); keeps what `backward` needs."""
        y, stream, mean, rstd = block.layer_norm_fwd(x, self.norm_weight, self.norm_bias, self.eps, residual=stream)
        self._kept = (y, stream, mean, rstd)
        return self.training.fwd(y, self.Wgu, self.Wd), stream

    def backward(self, dx, dstream):
        """Gradient of x and of stream (they enter as a sum: one tensor), and of the weights: (d, [dnorm_weight, dnorm_bias, dWgu, dWd])."""
        y, stream, mean, rstd = self._kept
        dy, dWgu, dWd = self.training.bwd(dx, y, self.Wgu, self.Wd)
        d, dweight, dbias = block.layer_norm_bwd(dy, stream, self.norm_weight, mean, rstd, dS=dstream)
        return d, [dweight, dbias, dWgu, dWd]

    def step(self, grads, rate: float):
        """Each weight moves by `rate` of its norm against its gradient."""
        for p, g in zip((self.norm_weight, self.norm_bias, self.Wgu, self.Wd), grads):
            p.sub_((rate * p.float().norm().clamp(min=1.0) / g.float().norm().clamp(min=1e-20) * g).to(p.dtype))

    def serve(self, x, stream, int8=None):
        """forward without a backward; int8: the context that `quantised` made."""
        y, stream, _, _ = block.layer_norm_fwd(x, self.norm_weight, self.norm_bias, self.eps, residual=stream)
        return (self.serving.fwd(y, self.Wgu, self.Wd) if int8 is None else int8.fwd(y)), stream

    def quantised(self) -> block.GatedI8Context:
        """The present weights in int8."""
        return block.GatedI8Context(self.T, self.Wgu, self.Wd, act=self.act)


def main(T: int = 1000, D: int = 512, F: int = 1408, steps: int = 30):
    g = torch.Generator(device="cuda").manual_seed(1)
    x, stream, target = ((torch.randn((T, D), generator=g, device="cuda") * s).to(torch.bfloat16) for s in (0.5, 1.0, 1.0))
    layers = [GatedSublayer(T, D, F, seed=i) for i in range(2)]
    for step in range(steps):
        a, s = x, stream
        for layer in layers:
            a, s = layer.forward(a, s)
        error = a.float() + s.float() - target.float()
        d = (2.0 / D * error).to(torch.bfloat16)
        da, ds = d, d                                   # x' and stream' of the last sublayer are added up
        grads = []
        for layer in reversed(layers):
            da, g_layer = layer.backward(da, ds)
            ds = da
            grads.append(g_layer)
        for layer, g_layer in zip(reversed(layers), grads):
            layer.step(g_layer, 0.02)
        if step % 10 == 0 or step == steps - 1:
            print(f"step {step}: mean squared error {float((error * error).mean()):.4f}", flush=True)
    int8 = [layer.quantised() for layer in layers]
    for t in range(3):                                  # one token at a time
        outs = []
        for contexts in ([None] * len(layers), int8):
            a, s = x[t:t + 1], stream[t:t + 1]
            for layer, c in zip(layers, contexts):
                a, s = layer.serve(a, s, c)
            outs.append(a.float() + s.float())
        print(f"token {t}: int8 differs from bf16 by {float((outs[1] - outs[0]).norm() / outs[0].norm()):.2%}", flush=True)


if __name__ == "__main__":
    main()
