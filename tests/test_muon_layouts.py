"""Which layouts of weights and momentum Muon takes beside S[din, dout]."""
import pytest
import torch

import paper_2510_00236_amd as pex

P = pex.MuonParams(lr=0.02, nesterov=1)
# of S [12, 20]
SAME = [(240,), (12, 20), (12, 4, 5), (3, 4, 20), (3, 4, 4, 5), (1, 12, 20)]
OTHER = [(20, 12), (24, 10), (6, 40), (20, 3, 4), (5, 48), (240, 1)]


@pytest.mark.parametrize("which", [0, 1])
def test_another_matrix_of_as_many_elements_is_refused(which):
    S = torch.zeros(12, 20)
    for shape in OTHER:
        t = [torch.zeros(240), torch.zeros(240), S]
        t[which] = torch.zeros(shape)
        with pytest.raises(ValueError, match="lie as S"):
            pex.pex_muon_step([t], P)
    for shape in SAME:          # (what is not refused for its shape is for where it lives)
        t = [torch.zeros(240), torch.zeros(240), S]
        t[which] = torch.zeros(shape)
        with pytest.raises(ValueError, match="GPU memory"):
            pex.pex_muon_step([t], P)


def test_vectors_lie_the_same_both_ways():
    for s, t in (((1, 7), (7, 1)), ((7, 1), (1, 7)), ((7, 1), (7, 1)), ((1, 7), (1, 1, 7))):
        with pytest.raises(ValueError, match="GPU memory"):
            pex.pex_muon_step([(torch.zeros(t), torch.zeros(t), torch.zeros(s))], P)


@pytest.mark.gpu
def test_the_same_update_in_every_layout():
    g = torch.Generator(device="cuda").manual_seed(1)
    theta, m, S = (torch.randn(12, 20, device="cuda", generator=g) for _ in range(3))
    want = None
    for shape in SAME:
        a, b = theta.clone().view(shape), m.clone().view(shape)
        pex.pex_muon_step([(a, b, S)], P)
        found = (a.view(12, 20), b.view(12, 20))
        want = want or found
        assert torch.equal(found[0], want[0]) and torch.equal(found[1], want[1])
    assert not torch.equal(want[0], theta)
