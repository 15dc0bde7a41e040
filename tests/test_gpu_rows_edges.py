"""Norms of rows at the ends of float32's range, refusals, and operators whose inputs are
read past the caches, in float32 and with a residual (MI355X only)."""
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


@pytest.mark.parametrize("d", [2, 3, 7, 64, 300])
def test_layer_norm_of_large_variance_and_eps(d):
    """A variance and an eps that float32 holds, whose sum it does not."""
    eps, half = 3.4e38, d // 2
    a = (2.9e38 / (2 * half)) ** 0.5                         # (the sum of squares, 2.9e38, is in range too)
    x = torch.zeros(4, d)
    x[:, :half], x[:, half:2 * half] = a, -a
    x[2] *= 1e-19
    x, dy = x.cuda(), rows(4, d, F32, seed=2)
    want, bound = rh.layer_norm(x, None, None, eps, F32)
    within(mol.layer_norm(x, eps=eps), want, bound, "y")
    (dx, dgamma, _), (bx, bg, _) = rh.layer_norm_grad(dy, x, None, eps, F32)
    got = mol.layer_norm_grad(dy, x, eps=eps)
    within(got[0], dx, bx, "dx")
    within(got[1], dgamma, bg, "dgamma")


@pytest.mark.parametrize("d", [9, 64, 300, 5000])
@pytest.mark.parametrize("to", [F32, BF16])
def test_gradients_of_rows_as_large_as_float32_holds(d, to):
    """1 / |x| is below float32's normal numbers, dy / |x| is not."""
    x, dy = rows(5, d, F32), rows(5, d, F32, seed=2)
    x = x / x.abs().amax(1, keepdim=True)
    x[1] *= 3e38
    x[3] *= 1.5e38
    dy *= 1e30
    want, bound = rh.normalize_grad(dy, x, 1e-12, to)
    within(mol.normalize_grad(dy, x, dtype=to), want, bound, "unit rows")
    (want, _, _), (bound, _, _) = rh.layer_norm_grad(dy, x, None, 1e-5, to)
    within(mol.layer_norm_grad(dy, x, dtype=to)[0], want, bound, "layer norm")
    # and the smallest: |x| of 2^-60 and below, of dy far smaller and larger than it
    x[1] = x[1] * 2.0 ** -128 * 1e-30
    x[3] = x[3] * 2.0 ** -128 * 2.0 ** -60
    for scale in (1e-60, 1e-25):
        small = dy * scale
        want, bound = rh.normalize_grad(small, x, 1e-37, to)
        within(mol.normalize_grad(small, x, eps=1e-37, dtype=to), want, bound + 1e-44, f"unit rows, dy of {scale}")


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64])
def test_output_types_are_refused_with_an_output_too(dtype):
    x = torch.zeros(3, 8, device="cuda")
    out = torch.full((3, 8), 7.0, dtype=dtype, device="cuda")
    for call in (lambda **k: mol.layer_norm(x, **k), lambda **k: mol.normalize(x, **k), lambda **k: mol.normalize_grad(x, x, **k),
                 lambda **k: mol.layer_norm_grad(x, x, **k), lambda **k: mol.dropout(x, 0.5, 1, **k), lambda **k: mol.gated_scan(x, x, **k),
                 lambda **k: mol.gated_step(x, x, x.clone(), **k)):
        for given in (dict(dtype=dtype), dict(out=out), dict(dtype=dtype, out=out)):
            with pytest.raises(ValueError, match="dtype"):
                call(**given)
    assert bool((out == 7).all())


@pytest.mark.parametrize("T,d", [(70001, 512), (300007, 131)])
def test_float32_norms_back_past_the_caches(T, d):
    """256 MB and more of float32 rows: rows as they are alone, and the weights' sums."""
    assert T * d * 8 >= 1 << 28
    g = torch.Generator(device="cuda").manual_seed(7)
    x, dy = (torch.randn(T, d, generator=g, device="cuda") for _ in range(2))
    some = [0, 1, T // 2, T - 2, T - 1]
    xs, ds = x[some].contiguous(), dy[some].contiguous()
    dx, dgamma, dbeta = mol.layer_norm_grad(dy, x)
    (want, _, _), (bound, _, _) = rh.layer_norm_grad(ds, xs, None, 1e-5, F32)
    within(dx[some], want, bound, "dx")
    assert torch.equal(dx[some], mol.layer_norm_grad(ds, xs)[0])
    unit = mol.normalize_grad(dy, x)
    within(unit[some], *rh.normalize_grad(ds, xs, 1e-12, F32), "dx of unit rows")
    assert torch.equal(unit[some], mol.normalize_grad(ds, xs))
    c = x.double() - x.double().mean(1, keepdim=True)
    xhat = c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt()
    # a lane's rows are at most T / 1024 of a workgroup's, then 6 additions over lanes, 3 over waves, 80 over workgroups;
    # xhat is off by 2 PATH U of its row's largest at most
    n = T / 1024 + 128
    within(dbeta, dy.double().sum(0), n * rh.U * dy.double().abs().sum(0), "dbeta")
    within(dgamma, (dy * xhat).sum(0), (n + 2 * rh.PATH) * rh.U * dy.double().abs().sum(0) * float(xhat.abs().max()), "dgamma")


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("p", [0.3, 0.9])
def test_dropout_with_residual_past_the_caches(t, p):
    n = (1 << 28) // (2 * (4 if t == F32 else 2)) + 16003
    g = torch.Generator(device="cuda").manual_seed(8)
    x, res = (torch.empty(n, dtype=t, device="cuda").normal_(generator=g) for _ in range(2))
    got = mol.dropout(x, p, 5, step=3, offset=1 << 33, residual=res)
    for at in (0, n // 16 * 8, n // 8 * 8 - 4000):
        piece = slice(at, min(at + 5000, n))
        _, want, bound = rh.dropout(x[piece], p, 5, 3, (1 << 33) + at, res[piece], t)
        # (of a sum that cancels, the bound counts the terms)
        within(got[piece], want, bound + 3 * rh.U * (x[piece].double().cpu().abs() / (1 - p) + res[piece].double().cpu().abs()), f"at {at}")
    assert torch.equal(mol.dropout(x, p, 5, step=3, offset=1 << 33, residual=res, out=res), got), "in place differs"
