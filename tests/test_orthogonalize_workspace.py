"""What the workspace queries of orthogonalisation and Muon ask for is what a call uses."""
import pytest
import torch

import paper_2510_00236_amd as pex


def test_small_matrices_need_none():
    q = pex.pex_orthogonalize_workspace_bytes
    for rows, cols in ((1, 1), (16, 16), (64, 256), (100, 128), (1, 256)):
        for dt in (pex.PEX_F32, pex.PEX_BF16):
            assert q(1, rows, cols, dt) == q(100000, rows, cols, dt) == 256
    assert q(1, 129, 128, 0) > 4 * 3 * 129 * 128 and q(3, 129, 128, 0) == 3 * q(1, 129, 128, 0)


def test_muon_asks_for_what_is_taken_at_a_time():
    q = pex.pex_muon_step_workspace_bytes
    one = q([(768, 768)])
    assert q([(768, 768)] * 24) == 24 * one == q([(768, 768)] * 48) == q([(768, 768)] * 49)
    # the largest of the groups, in the order of the array
    assert q([(768, 768)] * 24 + [(2048, 2048)]) == max(24 * one, q([(2048, 2048)]))
    assert q([(8, 8)] * 20) <= 20 * 256


@pytest.mark.gpu
def test_a_model_through_the_memory_that_is_asked_for():
    """Forty tensors of several sizes, and no byte past the workspace is touched."""
    shapes = [(300, 200), (64, 64), (768, 768), (40, 900), (1, 33)] * 8
    p = pex.MuonParams(lr=0.02)
    g = torch.Generator(device="cuda").manual_seed(1)
    S = [torch.randn(s, device="cuda", generator=g) for s in shapes]
    theta = [torch.randn(s, device="cuda", generator=g) for s in shapes]
    runs = []
    need = pex.pex_muon_step_workspace_bytes(shapes)
    for room in (need, 4 * need):
        buf = torch.full((room + 4096,), 171, dtype=torch.uint8, device="cuda")
        tensors = [(t.clone(), torch.zeros_like(t), s) for t, s in zip(theta, S)]
        pex.pex_muon_step(tensors, p, workspace=buf[:room])
        assert (buf[room:] == 171).all()
        runs.append(tensors)
    for a, b in zip(*runs):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.isfinite(a[0]).all()


@pytest.mark.gpu
def test_many_small_matrices_without_a_workspace():
    M = torch.randn(20000, 16, 16, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    torch.cuda.synchronize()
    pex.pex_orthogonalize(M[:1])
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    O = pex.pex_orthogonalize(M)
    # the result (an allocation's size goes by whole 2 MiB) and nothing of that size beside it
    assert torch.cuda.max_memory_allocated() - before <= O.numel() * 4 + (2 << 20)
    assert torch.equal(O[19999], pex.pex_orthogonalize(M[19999].clone()))
