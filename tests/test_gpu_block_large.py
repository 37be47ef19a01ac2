"""The operators around the block on tensors beyond 4 GiB, where an offset of 32 bits would wrap, and the norm's kernels for tensors that no cache holds.

A row's result does not depend on the rows beside it.  The norm and the int8 products have to give the bits of a small call on the same rows (what those are is
tested against 64 bits elsewhere); the bf16 block, whose tiles differ with the size, is held to its definition row by row, and its weight gradients as sums over chunks of tokens."""
import pytest
import torch

from paper_2503_16672_amd import block
from test_gpu_gated import U, check, reference
from test_gpu_norm import U as U32

BF16, F32 = torch.bfloat16, torch.float32


def _rand(shape, seed, dtype=BF16, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(shape, dtype=dtype, device="cuda")
    for rows in out.split(max(1, (1 << 28) // shape[1])):        # (the generator draws fp32)
        rows.copy_(torch.randn(rows.shape, generator=g, device="cuda") * scale)
    return out


# rows of each number of waves with the streaming hint (128 MiB and more), in both types; the last two beyond 4 GiB
@pytest.mark.gpu
@pytest.mark.parametrize("T,D,dtype", [(150001, 448, BF16), (70001, 1000, BF16), (40001, 2048, F32), (20001, 4096, BF16), (10001, 8192, F32), (4101, 16384, BF16), (270001, 8000, BF16), (1100001, 1001, F32)])
def test_norm(T, D, dtype):
    X, R, dY, dS = (_rand((T, D), s, dtype) for s in range(4))
    w, b = 1 + 0.3 * _rand((1, D), 5, F32)[0], _rand((1, D), 6, F32)[0]
    Y, S, mean, rstd = block.layer_norm_fwd(X, w, b, residual=R)
    dX, dw, db = block.layer_norm_bwd(dY, S, w, mean, rstd, dS=dS)
    step = 1 << 16 if T > 200000 else 1 << 12
    sums = [torch.zeros(D, dtype=torch.float64, device="cuda") for _ in range(4)]
    for i in range(0, T, step):
        j = min(i + step, T)
        if T <= 200000 or i == 0 or j == T or (i // step) % 3 == 0:
            few = 1000                                           # (rows that need no hint)
            for k in (i, max(i, j - few)):
                part = slice(k, min(k + few, j))
                y, s, m, r = block.layer_norm_fwd(X[part].contiguous().clone(), w, b, residual=R[part].clone())
                assert all(torch.equal(p, q[part]) for p, q in ((y, Y), (s, S), (m, mean), (r, rstd)))
                assert torch.equal(block.layer_norm_bwd(dY[part].clone(), s, w, m, r, dS=dS[part].clone())[0], dX[part])
        dy = dY[i:j].double()
        xh = (S[i:j].double() - mean[i:j, None].double()) * rstd[i:j, None].double()
        for total, term in zip(sums, (dy * xh, dy, (dy * xh).abs(), dy.abs())):
            total += term.sum(dim=0)
    # a sum over T tokens in workgroups' rows, then over the workgroups: at most T / 256 + 512 additions one after the other
    tol = (T / 256 + 512) * U32
    assert bool(((dw.double() - sums[0]).abs() <= tol * sums[2]).all()) and bool(((db.double() - sums[1]).abs() <= tol * sums[3]).all())


@pytest.mark.gpu
def test_gated_block_beyond_4_gib():
    T, D, F, act = 70001, 64, 16384, "gelu"                      # (G, U and their gradients: 4.6 GB each)
    X, Wgu, Wd, dY = _rand((T, D), 1), _rand((D, 2 * F), 2, scale=D ** -0.5), _rand((F, D), 3, scale=F ** -0.5), _rand((T, D), 4)
    ctx = block.GatedContext(T, D, F, act=act, training=True)
    Y = ctx.fwd(X, Wgu, Wd)
    dX, dWgu, dWd = ctx.bwd(dY, X, Wgu, Wd)
    sums = {n: [torch.zeros(t.shape, dtype=torch.float64, device="cuda") for _ in range(2)] for n, t in (("dWgu", dWgu), ("dWd", dWd))}
    for i in range(0, T, 5000):
        part = slice(i, min(i + 5000, T))
        ref = reference(X[part], Wgu, Wd, dY[part], act)
        check(Y[part], ref["Y"], "Y")
        check(dX[part], ref["dX"], "dX")
        for n, (out, squares) in sums.items():                   # sigma^2 = U^2 / 3 (squares of the products + output^2)
            out += ref[n][0]
            squares += ref[n][1] ** 2 * 3 / U ** 2 - ref[n][0] ** 2
    for n, got in (("dWgu", dWgu), ("dWd", dWd)):
        out, squares = sums[n]
        check(got, (out, U / 3 ** 0.5 * torch.sqrt(squares + out ** 2)), n)
    serving = block.GatedContext(T, D, F, act=act)
    assert torch.equal(serving.fwd(X, Wgu, Wd), Y)


@pytest.mark.gpu
def test_int8_beyond_4_gib():
    T, D, F = 140003, 64, 16384                                  # (Y of the product and the block's h: 4.6 GB)
    X, Wgu, Wd = _rand((T, D), 1), _rand((D, 2 * F), 2, scale=D ** -0.5), _rand((F, D), 3, scale=F ** -0.5)
    W8 = block.I8Weight(_rand((D, F), 4, scale=D ** -0.5))
    large, small = block.GatedI8Context(T, Wgu, Wd), block.GatedI8Context(3000, Wgu, Wd)
    Y, Z = large.fwd(X), block.linear_i8(X, W8)
    codes, scales = block.quantise_i8(X)
    assert torch.equal(block.matmul_i8(codes, scales, W8), Z)
    for i in range(0, T, 3000):
        part = X[i:i + 3000].clone()
        assert torch.equal(small.fwd(part), Y[i:i + 3000]), i
        assert torch.equal(block.linear_i8(part, W8), Z[i:i + 3000]), i


@pytest.mark.gpu
def test_wide_rows_beyond_4_gib_to_codes():
    T, K = 20001, 1 << 17                                        # (5.2 GB of tokens)
    X = _rand((T, K), 1)
    codes, scales = block.quantise_i8(X)
    for i in range(0, T, 1000):
        c, s = block.quantise_i8(X[i:i + 1000].clone())
        assert torch.equal(c, codes[i:i + 1000]) and torch.equal(s, scales[i:i + 1000])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 1030])
def test_codes_of_the_smallest_values(T):
    """Tokens around and below the smallest normal bf16: scales and quotients are subnormal fp32 values and are not flushed."""
    X = _rand((T, 64), 1)
    X = (X.cpu().float() * torch.logspace(-41, -35, T)[:, None]).to(BF16)
    codes, scales = block.quantise_i8(X.cuda())
    top = X.float().abs().amax(dim=1, keepdim=True)
    s = torch.where(top > 0, top * (1.0 / 127.0), torch.ones_like(top))
    assert torch.equal(scales.cpu(), s[:, 0])
    live = s[:, 0] > 0
    assert torch.equal(codes.cpu()[live].float(), torch.round(X.float() / s).clamp(-127, 127)[live])
