"""Layer norm over more rows, examples and columns than one launch has places for: rows do not depend on each other, so that the whole
is, to the bit, what its parts are."""
import pytest
import torch

import paper_2510_00236_amd as pex

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def rand(shape, dtype, seed):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed), dtype=torch.float32).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [1, 3])
def test_many_narrow_rows(d, dtype):
    """More than 2^22 rows of less than 16 bytes."""
    B, T = 2, (1 << 21) + 3
    X, G = rand((B, T, d), dtype, 1), rand((B, T, d), dtype, 2)
    gamma, beta = 1 + 0.2 * rand((d,), torch.float32, 3), rand((d,), torch.float32, 4)
    Y, mean, rstd = pex.pex_layer_norm(X, gamma, beta)
    dX, stats = pex.pex_layer_norm_grad(G, X, mean, rstd, gamma, want=("identity", "square"))
    alone, _ = pex.pex_layer_norm_grad(G, X, mean, rstd, gamma, want=())
    assert torch.equal(alone, dX)
    for b in range(B):
        for lo, hi in ((0, T // 2), (T // 2, T)):
            x, g = X[b, lo:hi].contiguous()[None], G[b, lo:hi].contiguous()[None]
            y, m, r = pex.pex_layer_norm(x, gamma, beta)
            assert torch.equal(y[0], Y[b, lo:hi]) and torch.equal(m[0], mean[b, lo:hi]) and torch.equal(r[0], rstd[b, lo:hi])
            assert torch.equal(pex.pex_layer_norm_grad(g, x, m, r, gamma, want=())[0][0], dX[b, lo:hi])
    xh = (X.double() - mean.double()[..., None]) * rstd.double()[..., None]
    for name, terms in (("scale", G.double() * xh), ("offset", G.double())):
        v, size = terms.sum(1), terms.abs().sum(1) * (T + 16) * U       # a chain of T additions; the terms' own three roundings
        assert ((stats[name]["identity"].double() - v.sum(0)).abs() <= size.sum(0) + 4 * U * v.abs().sum(0)).all()
        assert ((stats[name]["square"].double() - (v * v).sum(0)).abs() <= (2 * v.abs() * size + size * size).sum(0) + 8 * U * (v * v).sum(0)).all()


@pytest.mark.parametrize("T,d,B", [(1, 8, (1 << 24) + 3), (3, 4, (1 << 24) + 1)])
def test_many_examples_without_statistics(T, d, B):
    dtype = torch.bfloat16 if d == 8 else torch.float32
    X, G = rand((B, T, d), dtype, 5), rand((B, T, d), dtype, 6)
    gamma = 1 + 0.2 * rand((d,), torch.float32, 7)
    mean, rstd = X.float().mean(2), torch.rsqrt(X.float().var(2, correction=0) + 1e-5)
    dX, stats = pex.pex_layer_norm_grad(G, X, mean, rstd, gamma, want=())
    assert stats == {"scale": {}, "offset": {}}
    for lo in (0, B // 2, B - 5000):
        at = slice(lo, lo + 5000)
        part, _ = pex.pex_layer_norm_grad(G[at], X[at], mean[at], rstd[at], gamma, want=())
        assert torch.equal(part, dX[at])


def test_a_row_of_half_a_billion_columns():
    """Statistics of two vectors that are more blocks of columns than one launch of their second pass holds."""
    d = (1 << 29) + 5
    X, G = (torch.empty(1, 2, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t, seed in ((X, 8), (G, 9)):
        for row in t[0]:
            row.copy_(rand((1 << 16,), torch.bfloat16, seed).repeat((d >> 16) + 1)[:d])      # what is drawn once, over and over
            seed += 2
    mean, rstd = torch.tensor([[0.25, -0.5]], device="cuda"), torch.tensor([[1.5, 0.75]], device="cuda")
    dX, stats = pex.pex_layer_norm_grad(G, X, mean, rstd, want=("identity",), dX=torch.empty_like(G))
    assert torch.isfinite(dX).all()
    period = 1 << 16
    for at in (0, (1 << 28) - period, 1 << 28, (1 << 29) - period, d - period):
        g, x = (t[0, :, at:at + period].double() for t in (G, X))
        xh = (x - mean[0].double()[:, None]) * rstd[0].double()[:, None]
        for name, terms in (("scale", g * xh), ("offset", g)):
            got = stats[name]["identity"][at:at + period].double()
            assert ((got - terms.sum(0)).abs() <= 8 * U * (g.abs() * (x.abs() + 1)).sum(0) * 1.5).all(), (name, at)
    # everywhere: the sum of the offset is that of the row
    assert torch.equal(stats["offset"]["identity"][period:2 * period], stats["offset"]["identity"][:period])
    whole = stats["offset"]["identity"][: d - 5].view(-1, period)
    assert torch.equal(whole, whole[:1].expand_as(whole))
