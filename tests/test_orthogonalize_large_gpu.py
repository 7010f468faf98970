"""Orthogonalisation on the kernels of many blocks (256 x 256 through LDS, and four slots of 128 x 128 in an update) and two steps at a time through
the Gram matrix with every number of steps.  Which kernels these sizes are on test_orthogonalize_plan_host.py asks.

The exact result in 64 bits on the GPU; the bar of fp32 matrices is that of test_orthogonalize_gpu.py, a bf16 result's is its rounding's and twice
that (test_orthogonalize_rounding_gpu.py)."""
import math

import pytest
import torch

import paper_2510_00236_amd as pex

pytestmark = pytest.mark.gpu

BAR = 5e-6
DEFAULT = (3.4445, -4.7750, 2.0315)


def rand(shape, seed):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def noisy(rows, cols, seed):
    r = min(3, rows, cols)
    top = 4.0 * (math.sqrt(rows) + math.sqrt(cols)) / math.sqrt(rows * cols)
    return rand((rows, cols), seed) + top * rand((rows, r), seed + 1000) @ rand((r, cols), seed + 2000)


def exact(M, steps=5, coefficients=DEFAULT, eps=1e-7):
    """By way of the Gram matrix of the shorter side: all factors are polynomials of it"""
    a, b, c = coefficients
    X = M.double()
    tall = X.shape[0] > X.shape[1]
    X = X.t().contiguous() if tall else X
    X = X / (X.norm() + eps)
    W = torch.mm(X, X.t().contiguous())
    unit = torch.eye(W.shape[0], dtype=torch.float64, device="cuda")
    Q = unit
    for _ in range(steps):
        F = a * unit + b * W + c * torch.mm(W, W)
        Q = torch.mm(F, Q)
        W = torch.mm(F, torch.mm(W, F))
    O = torch.mm(Q, X)
    return O.t() if tall else O


def assert_near(got, want, dtype=torch.float32):
    own = float(torch.norm(want.to(dtype).double() - want)) if dtype == torch.bfloat16 else 0.0
    bar = BAR * float(torch.norm(want))
    assert float(torch.norm(got.double() - want)) <= own + (2 * bar if own else bar)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("count,rows,cols", [(1, 2048, 8192), (1, 8192, 2048), (1, 2000, 8190), (7, 2048, 2048), (1, 5376, 5400)])
def test_blocks_of_256(count, rows, cols, dtype):
    M = torch.stack([noisy(rows, cols, 3 * i) for i in range(count)]).to(dtype)
    O = pex.pex_orthogonalize(M)
    for i in {0, count - 1}:
        assert_near(O[i], exact(M[i]), dtype)
    code = pex.PEX_F32 if dtype == torch.float32 else pex.PEX_BF16
    ws = torch.empty(pex.pex_orthogonalize_workspace_bytes(1, rows, cols, code), dtype=torch.uint8, device="cuda").fill_(255)
    assert torch.equal(O, pex.pex_orthogonalize(M, workspace=ws)) and torch.equal(O, pex.pex_orthogonalize(M, out=M, workspace=ws))


@pytest.mark.parametrize("shapes", [[(2048, 8192), (8192, 2048)], [(2304, 2304)], [(2048, 2048)] * 7])
def test_updates(shapes):
    p = pex.MuonParams(lr=0.02, momentum=0.9, weight_decay=1e-3, nesterov=1, scaling=pex.PEX_MUON_SCALE_RMS)
    start = [(0.02 * rand(s, k), noisy(*s, 10 + k), noisy(*s, 20 + k)) for k, s in enumerate(shapes)]
    tensors = [(t.clone(), m.clone(), S) for t, m, S in start]
    pex.pex_muon_step(tensors, p)
    beta = float(p.momentum)
    for k in {0, len(shapes) - 1}:
        (theta, m, S), (got, got_m, _) = start[k], tensors[k]
        want_m = beta * m.double() + (1 - beta) * S.double()
        assert ((got_m.double() - want_m).abs() <= 3 * 2.0 ** -24 * (m.double().abs() + S.double().abs())).all()
        O = exact(beta * want_m + (1 - beta) * S.double())
        step = float(p.lr) * 0.2 * math.sqrt(max(theta.shape))
        want = theta.double() - step * O - float(p.weight_decay) * theta.double()
        assert torch.norm(got.double() - want) <= step * BAR * O.norm() + 4 * 2.0 ** -24 * torch.norm(want.abs() + theta.double().abs())


# a larger bound where steps leave more of the small singular values' growth a^k to come: see the bound of test_orthogonalize_gpu.py, which goes by it
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7])
@pytest.mark.parametrize("coefficients", [DEFAULT, (1.875, -1.25, 0.375), (1.5, -0.5, 0.0)])
@pytest.mark.parametrize("rows,cols", [(520, 1000), (1900, 600), (1024, 1600)])
def test_steps_through_the_gram_matrix(rows, cols, steps, coefficients):
    M = noisy(rows, cols, steps)
    p = pex.NewtonSchulzParams(*coefficients, steps=steps)
    assert_near(pex.pex_orthogonalize(M, params=p), exact(M, steps, coefficients))
