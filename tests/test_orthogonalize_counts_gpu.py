"""More small matrices than one launch has places for: the whole is, to the bit, what its parts are."""
import pytest
import torch

import paper_2510_00236_amd as pex

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_eight_million_scalars(dtype):
    count = (1 << 23) + 5
    M = torch.randn(count, 1, 1, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(dtype)
    M[::1000] = 0
    p = pex.NewtonSchulzParams(steps=1)
    code = pex.PEX_F32 if dtype == torch.float32 else pex.PEX_BF16
    ws = torch.empty(pex.pex_orthogonalize_workspace_bytes(1, 1, 1, code), dtype=torch.uint8, device="cuda")
    O = pex.pex_orthogonalize(M, out=torch.full_like(M, 99.0), params=p, workspace=ws)
    for lo in range(0, count, 1 << 21):
        part = M[lo:lo + (1 << 21)]
        assert torch.equal(O[lo:lo + (1 << 21)], pex.pex_orthogonalize(part, params=p, workspace=ws)), lo
    assert (O[::1000] == 0).all() and (O.abs() < 2).all()
