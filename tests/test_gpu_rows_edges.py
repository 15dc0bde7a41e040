"""Norms of rows whose sums leave float32's range (MI355X only)."""
import pytest
import torch

import rows_helpers as rh
from learn_helpers import within
from paper_2407_15462_amd import mol
from test_gpu_rows import rows

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("d", [2, 8, 9, 64, 300, 1024, 5000, 16384])
@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_layer_norm_of_constant_rows_whose_sum_overflows(d, t, sign):
    """Mean 2^127, variance 0: y is beta, and dx = (w - mean(w)) / sqrt(eps); beside ordinary rows."""
    x, dy = rows(5, d, t), rows(5, d, F32, seed=2)
    big = sign * 2.0 ** 127
    x[1] = big
    x[3] = big
    g = torch.Generator().manual_seed(d)
    gamma, beta = (1 + 0.3 * torch.randn(d, generator=g)).cuda(), torch.randn(d, generator=g).cuda()
    y = mol.layer_norm(x, gamma, beta, dtype=F32)
    assert torch.equal(y[1], beta) and torch.equal(y[3], beta)
    small = x.clone()
    small[1], small[3] = 0, 0                                # (a row of zeros: the same variance, and the same xhat)
    assert torch.equal(mol.layer_norm(small, gamma, beta, dtype=F32), y)
    got, want = mol.layer_norm_grad(dy, x, gamma, dtype=F32), mol.layer_norm_grad(dy, small, gamma, dtype=F32)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    (dx, dgamma, dbeta), bounds = rh.layer_norm_grad(dy, small, gamma, 1e-5, F32)
    for name, a, b, c in zip(("dx", "dgamma", "dbeta"), got, (dx, dgamma, dbeta), bounds):
        within(a, b, c, name)
