"""bf16 matrices are orthogonalised as exactly as fp32 ones, and the result is rounded once.

Let O be the exact result, F the kernels' before that rounding, round(F) what comes out.  round(F) is the nearest bf16 to F, so
|round(F) - F| <= |round(O) - F| <= |round(O) - O| + |O - F| entry by entry, and |round(F) - O| <= |round(O) - O| + 2 |O - F|.  |O - F| in the
2-norm is at most the bar of fp32 matrices, 5e-6 |O|."""
import numpy as np
import pytest
import torch

import paper_2510_00236_amd as pex

pytestmark = pytest.mark.gpu


def exact(M, steps=5, a=3.4445, b=-4.7750, c=2.0315, eps=1e-7):
    X = M.double().numpy()
    tall = X.shape[0] > X.shape[1]
    X = X.T if tall else X
    X = X / (np.linalg.norm(X) + eps)
    for _ in range(steps):
        A = X @ X.T
        X = a * X + (b * A + c * A @ A) @ X
    return X.T if tall else X


# straight from the caches and through LDS, one workgroup, thin, tall, ragged, many at once, two steps through the Gram matrix
@pytest.mark.parametrize("count,rows,cols", [(1, 100, 90), (1, 40, 900), (3, 257, 129), (12, 768, 768), (1, 1002, 300), (2, 1600, 520), (2, 1100, 1100), (40, 192, 320)])
def test_bf16_results_are_off_by_their_rounding(count, rows, cols):
    g = torch.Generator().manual_seed(rows + cols)
    M = (torch.randn(count, rows, cols, generator=g) + 0.5 * torch.randn(count, rows, 2, generator=g) @ torch.randn(count, 2, cols, generator=g)).bfloat16()
    got = pex.pex_orthogonalize(M.cuda()).cpu().double().numpy()
    for i in {0, count - 1}:
        want = exact(M[i])
        own = np.linalg.norm(torch.from_numpy(want).bfloat16().double().numpy() - want)
        assert np.linalg.norm(got[i] - want) <= own + 2 * 5e-6 * np.linalg.norm(want), np.linalg.norm(got[i] - want) / own
