"""Muon over matrices that different kernels take in the same round: blocks of 256 and 128 beside sides that only smaller ones divide."""
import math

import pytest
import torch

import paper_2510_00236_amd as pex

pytestmark = pytest.mark.gpu

# the fp32 bar of test_orthogonalize_gpu.py
BAR = 5e-6


def exact(u, a=3.4445, b=-4.7750, c=2.0315, steps=5, eps=1e-7):
    """In 64 bits, on the GPU"""
    X = u.t().contiguous() if u.shape[0] > u.shape[1] else u
    X = X / (X.norm() + eps)
    for _ in range(steps):
        A = torch.mm(X, X.t().contiguous())
        X = a * X + torch.mm(b * A + c * torch.mm(A, A), X)
    return X.t() if u.shape[0] > u.shape[1] else X


@pytest.mark.parametrize("shapes", [[(1024, 1024)] * 8 + [(1024, 320), (1024, 40), (300, 1024), (64, 64)], [(2048, 2400), (320, 320), (2400, 2048), (2048, 10)],
                                    [(4096, 3800), (640, 640), (3800, 192)], [(2304, 2304), (320, 2304), (1152, 2304)]])
def test_mixed_sizes(shapes):
    p = pex.MuonParams(lr=0.02, momentum=0.9, weight_decay=1e-3, grad_scale=0.5, nesterov=1, scaling=pex.PEX_MUON_SCALE_RMS)
    g = torch.Generator(device="cuda").manual_seed(len(shapes))
    start = [tuple(torch.randn(s, device="cuda", generator=g) for _ in range(3)) for s in shapes]
    need = max(pex.pex_muon_step_workspace_bytes([s]) for s in shapes)
    runs = []
    for room in (need, need + need // 2, pex.pex_muon_step_workspace_bytes(shapes)):
        tensors = [(t.clone(), m.clone(), S) for t, m, S in start]
        pex.pex_muon_step(tensors, p, workspace=torch.empty(room, dtype=torch.uint8, device="cuda").fill_(255))
        runs.append(tensors)
    for a, b, c in zip(*runs):
        assert torch.equal(a[0], b[0]) and torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])
    beta = float(p.momentum)
    for (theta, m, S), (got, got_m, _) in zip(start, runs[0]):
        mu = S.double() * 0.5
        want_m = beta * m.double() + (1 - beta) * mu
        assert ((got_m.double() - want_m).abs() <= 3 * 2.0 ** -24 * (m.double().abs() + mu.abs())).all()
        O = exact(beta * want_m + (1 - beta) * mu)
        step = float(p.lr) * 0.2 * math.sqrt(max(theta.shape))
        want = theta.double() - step * O - float(p.weight_decay) * theta.double()
        assert torch.norm(got.double() - want) <= step * BAR * O.norm() + 4 * 2.0 ** -24 * torch.norm(want.abs() + theta.double().abs())
