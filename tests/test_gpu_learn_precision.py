"""What the learning operators keep of float32 (MI355X only)."""
import pytest
import torch

import learn_helpers as lh
from paper_2407_15462_amd import mol
from parity_helpers import log

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
NAMES = ("dQ", "dX", "da_q", "da_x", "dW1", "db1", "dW2", "db2")
SHAPES = [(5, 33, 4, 4, 64, 32), (9, 70, 8, 4, 64, 64), (6, 131, 8, 8, 32, 64), (7, 50, 3, 5, 40, 130), (4, 40, 8, 4, 128, 128),
          (13, 40, 8, 8, 31, 20)]


def thirds(g, dim):
    """g on the first of three equal rows, and -0.7 and -0.3 of it on the others: what all of them add up to is next to nothing."""
    return torch.cat([g, -0.7 * g, -0.3 * g], dim)


@pytest.mark.parametrize("B,N,Pq,Px,d,H", SHAPES)
def test_score_grad_in_float32_of_bf16_problems(B, N, Pq, Px, d, H):
    """MOL_FLAG_F32_GATING: sums whose terms cancel keep float32's precision until they are rounded to bf16.
    A pair's term takes about 20 float32 roundings, 2^-24 / sqrt(3) each in the root mean square, 2^-22.4 together; and
    three copies of a pair have the same ones up to the last few.  Terms kept in 16 bits are off by 2^-18.5 of themselves."""
    log(f"[score_grad f32] B={B} N={N} P={Pq}x{Px} d={d} H={H}")
    inputs, g = lh.mol_inputs(B, N, Pq, Px, d, H, BF16, seed=B + N)
    Q, X, a_q, a_x, W1, b1, W2, b2 = inputs
    for over, names in (("items", ("dQ", "dW1", "dW2")), ("queries", ("dX", "dW1", "dW2"))):
        if over == "items":
            wide = [Q, torch.cat([X] * 3, 1), a_q, torch.cat([a_x] * 3), W1, b1, W2, b2]
            g3 = thirds(g, 1)
            first = torch.cat([g, 0 * g, 0 * g], 1)
        else:
            wide = [torch.cat([Q] * 3), X, torch.cat([a_q] * 3), a_x, W1, b1, W2, b2]
            g3 = thirds(g, 0)
            first = torch.cat([g, 0 * g, 0 * g], 0)
        want = lh.score_grads([t.float() for t in wide], g3)[0]
        size = lh.score_grads([t.float() for t in wide], first.abs())[0]        # (terms of one sign for the most part)
        prob = mol.Problem(*(t.cuda() for t in wide), flags=mol.MOL_FLAG_F32_GATING)
        got = mol.score_grad(prob, g3.cuda())
        for n in names:
            err = float((got[n].double().cpu() - want[n]).norm())
            assert err < 2.0 ** -8 * float(want[n].norm()) + 2.0 ** -21 * float(size[n].norm()), (over, n, err / float(size[n].norm()))


@pytest.mark.parametrize("B,N,Pq,Px,d,H", SHAPES)
def test_score_grad_in_float32_is_one_rounding_off(B, N, Pq, Px, d, H):
    """Every output within the bounds of a float32 evaluation and one rounding to its type."""
    inputs, g = lh.mol_inputs(B, N, Pq, Px, d, H, BF16, seed=B * N)
    want, bound = lh.score_grads([t.float() for t in inputs], g)
    got = mol.score_grad(mol.Problem(*(t.cuda() for t in inputs), flags=mol.MOL_FLAG_F32_GATING), g.cuda())
    for n in NAMES:
        half = lh.HALF[got[n].dtype]
        lh.within(got[n], want[n], bound[n] + half * (1 + 2 * half) * want[n].abs(), n)


# ------------------------------------------------------------------ AdamW
@pytest.mark.parametrize("g0", [3e-20, 1e-19, 1e-18, 1e-17, 1e-15, 1e-3])
@pytest.mark.parametrize("eight", [False, True], ids=["f32states", "e4m3states"])
def test_adamw_of_the_smallest_second_moments(g0, eight):
    """Second moments below 2^-126 (gradients below 3e-18) keep their root: with a small eps the step is lr, not m / eps.
    v = 0.001 g g has three roundings and what underflow adds, 2^-150; its root half of that, and the step 16 more."""
    n, eps, b1, b2 = 700, 1e-30, 0.9, 0.999
    gen = torch.Generator().manual_seed(5)
    p = torch.randn(n, generator=gen)
    g = g0 * (1 + torch.rand(n, generator=gen)) * torch.where(torch.rand(n, generator=gen) < 0.5, -1.0, 1.0)
    zeros = lambda: torch.zeros(n, dtype=torch.float8_e4m3fn if eight else torch.float32, device="cuda")  # noqa: E731
    got, m, v = p.cuda(), zeros(), zeros()
    scales = [[torch.zeros(3, device="cuda")] for _ in range(2)] if eight else [None, None]
    mol.adamw_step(mol.AdamwTensors([got], [g.cuda()], [m], [v], *scales), lr=0.5, eps=eps)
    want, wm, wv = lh.adamw(p, g, torch.zeros(n), torch.zeros(n), 0.5, b1, b2, eps, 0.0, 1)
    rel = 2.0 ** -150 / wv + 20 * lh.U
    lh.within(got, want, (p.double() - want).abs() * rel + 2 * lh.U * (p.double().abs() + 0.5), "p")
    if eight:
        top = torch.stack([x.abs().max() for x in wv.sqrt().split(256)])
        lh.within(scales[1][0], top / 448, top * (2.0 ** -150 / wv.min() + 12 * lh.U), "scale of v")
        back = v.float().double().cpu() * scales[1][0].double().cpu().repeat_interleave(256)[:n]
        assert bool(((back / wv.sqrt() - 1).abs() <= 0.126).all()), "codes: a neighbour's distance is an eighth at most"
    else:
        lh.within(v, wv, wv * 4 * lh.U + 2.0 ** -150, "v")
