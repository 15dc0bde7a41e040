"""One workspace, kept for the largest calls of the learning operators, serves
smaller ones with the bits that a workspace of their own gives (MI355X only)."""
import pytest
import torch

import learn_helpers as lh
from paper_2407_15462_amd import mol
from parity_helpers import log

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def held(n):
    """n bytes of NaN between two bands of known ones."""
    buf = torch.full((n + 1024,), 0xFF, dtype=torch.uint8, device="cuda")
    buf[:512] = 0xA5
    buf[512 + n:] = 0xA5
    return buf, buf[512:512 + n]


def untouched(buf):
    return bool((buf[:512] == 0xA5).all()) and bool((buf[-512:] == 0xA5).all())


@pytest.mark.parametrize("Pq,Px,d,H,dtype,flags,sizes", [
    (8, 8, 64, 64, BF16, 0, [(1024, 2048), (568, 2048), (1024, 1137), (1024, 1100), (7, 2000), (3, 40), (1, 1)]),
    (8, 8, 64, 64, BF16, 1, [(300, 2048), (129, 2047), (4, 500), (3, 2048), (1, 33)]),
    (4, 4, 64, 32, F32, 0, [(200, 4000), (129, 3999), (16, 1024), (2, 4000), (1, 1)])])
def test_score_grad(Pq, Px, d, H, dtype, flags, sizes):
    kept, ws = None, None
    for B, N in sizes:
        log(f"[workspaces] score_grad {B} x {N} of {Pq}x{Px} {dtype}")
        inputs, dphi = lh.mol_inputs(B, N, Pq, Px, d, H, dtype, seed=B + N, device="cuda")
        prob = mol.Problem(*inputs, flags=flags)
        if ws is None:
            kept, ws = held(mol.mol_workspace_size(prob, mol.MOL_OP_SCORE_GRAD))
        got = mol.score_grad(prob, dphi, ws=ws)
        own = mol.score_grad(prob, dphi)
        assert all(torch.equal(got[n], own[n]) for n in own), (B, N)
    assert untouched(kept)


def test_embed_grad_and_loss():
    C, V, d = 1, 6040, 512
    kept, ws = held(mol.mol_embed_grad_workspace(C, V, d, 30000))
    for T in (30000, 16342, 8193, 8192, 3000, 20, 1):
        gen = torch.Generator().manual_seed(T)
        grad, ids = torch.randn(C, T, d, generator=gen).cuda(), torch.randint(-1, V, (T,), generator=gen).int().cuda()
        assert torch.equal(mol.embed_grad(grad, ids, V, ws=ws), mol.embed_grad(grad, ids, V)), T
    assert untouched(kept)
    kept, ws = held(mol.mol_softmax_loss_workspace(514, 40000))
    for B, N in ((514, 40000), (505, 40000), (128, 39999), (3, 34817), (2, 100)):
        gen = torch.Generator().manual_seed(B)
        phi, target = torch.randn(B, N, generator=gen).cuda(), torch.randint(0, N, (B,), generator=gen).int().cuda()
        got, want = mol.softmax_loss(phi, target, ws=ws), mol.softmax_loss(phi, target)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (B, N)
    assert untouched(kept)
