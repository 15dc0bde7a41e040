"""Refusals of the operators that learn the similarity: bad arguments are
turned down on the host, before anything is launched (CPU only)."""
import concurrent.futures as cf
import ctypes
import os

import pytest
import torch

from mfma_hazards import early_reads
from paper_2407_15462_amd import mol
from test_mfma_hazards import HIPCC, _asm

FAKE, BIG = 256, 1 << 40          # a pointer that is never followed; every call below stops before its launch
NAN = float("nan")


def _lookup(**kw):
    a = dict(table=FAKE, tt=mol.MOL_F32, C=2, V=10, d=8, ids=FAKE, T=5, scale=1.0, out=FAKE, ot=mol.MOL_BF16)
    a.update(kw)
    return mol.load().mol_embed_lookup(*a.values(), None)


@pytest.mark.parametrize("bad,status", [
    (dict(C=0), mol.MOL_EINVAL), (dict(V=0), mol.MOL_EINVAL), (dict(d=0), mol.MOL_EINVAL), (dict(T=-1), mol.MOL_EINVAL),
    (dict(C=65), mol.MOL_EUNSUPPORTED), (dict(d=65537), mol.MOL_EUNSUPPORTED), (dict(tt=2), mol.MOL_EUNSUPPORTED),
    (dict(ot=-1), mol.MOL_EUNSUPPORTED), (dict(table=None), mol.MOL_EINVAL), (dict(ids=None), mol.MOL_EINVAL),
    (dict(out=None), mol.MOL_EINVAL), (dict(T=1 << 30, d=8, C=2), mol.MOL_EUNSUPPORTED),
    (dict(V=(1 << 31) - 1, C=5), mol.MOL_EUNSUPPORTED),
])
def test_lookup_refuses(bad, status):
    assert _lookup(**bad) == status
    assert mol.load().mol_last_error()


def test_lookup_of_no_ids_needs_no_pointer():
    assert _lookup(T=0, table=None, ids=None, out=None) == mol.MOL_OK


def _grad(**kw):
    a = dict(grad=FAKE, gt=mol.MOL_F32, C=2, V=10, d=8, ids=FAKE, T=5, scale=1.0, acc=0, out=FAKE, ot=mol.MOL_BF16,
             ws=FAKE, n=BIG)
    a.update(kw)
    return mol.load().mol_embed_grad(*a.values(), None)


@pytest.mark.parametrize("bad,status", [
    (dict(C=0), mol.MOL_EINVAL), (dict(T=-1), mol.MOL_EINVAL), (dict(d=65537), mol.MOL_EUNSUPPORTED),
    (dict(gt=3), mol.MOL_EUNSUPPORTED), (dict(ot=3), mol.MOL_EUNSUPPORTED), (dict(acc=2), mol.MOL_EINVAL),
    (dict(grad=None), mol.MOL_EINVAL), (dict(ids=None), mol.MOL_EINVAL), (dict(out=None), mol.MOL_EINVAL),
    (dict(ws=None), mol.MOL_EINVAL), (dict(ws=FAKE + 8), mol.MOL_EINVAL), (dict(n=16), mol.MOL_EWORKSPACE),
])
def test_embed_grad_refuses(bad, status):
    assert _grad(**bad) == status


def test_embed_grad_sizes():
    assert _grad(T=0, acc=1, grad=None, ids=None, ws=None, out=None) == mol.MOL_OK     # nothing to add
    small, large = mol.mol_embed_grad_workspace(4, 1000, 64, 100), mol.mol_embed_grad_workspace(4, 1000, 64, 1 << 20)
    assert 0 < small < large and small % 256 == 0
    # every size up to a call's is served by that call's workspace
    last = 0
    for T in range(0, 9000, 37):
        n = mol.mol_embed_grad_workspace(8, 5000, 96, T)
        last = max(last, n)
        assert n <= mol.mol_embed_grad_workspace(8, 5000, 96, 20000)
    with pytest.raises(mol.MolError):
        mol.mol_embed_grad_workspace(0, 1, 1, 1)
    assert mol.load().mol_embed_grad_workspace(1, 1, 1, 1, None) == mol.MOL_EINVAL


def _loss(**kw):
    a = dict(B=4, N=10, phi=FAKE, target=FAKE, ids=None, inv_temp=1.0, w=None, loss=FAKE, dphi=FAKE, ws=None, n=0)
    a.update(kw)
    return mol.load().mol_softmax_loss(*a.values(), None)


@pytest.mark.parametrize("bad,status", [
    (dict(B=0), mol.MOL_EINVAL), (dict(N=0), mol.MOL_EINVAL), (dict(B=65536), mol.MOL_EUNSUPPORTED),
    (dict(phi=None), mol.MOL_EINVAL), (dict(target=None), mol.MOL_EINVAL), (dict(inv_temp=0.0), mol.MOL_EINVAL),
    (dict(inv_temp=-1.0), mol.MOL_EINVAL), (dict(inv_temp=NAN), mol.MOL_EINVAL),
    (dict(inv_temp=float("inf")), mol.MOL_EINVAL), (dict(N=100000), mol.MOL_EINVAL),
    (dict(N=100000, ws=FAKE, n=16), mol.MOL_EWORKSPACE),
])
def test_softmax_loss_refuses(bad, status):
    assert _loss(**bad) == status


def test_softmax_loss_without_outputs_is_nothing():
    assert _loss(loss=None, dphi=None) == mol.MOL_OK
    assert mol.mol_softmax_loss_workspace(4, 100) == 0 < mol.mol_softmax_loss_workspace(4, 100000)


def test_score_grad_refuses():
    lib = mol.load()
    c = mol.MolProblemC(4, 100, 2, 2, 64, 16, mol.MOL_BF16, *([FAKE] * 8))
    out = mol.MolScoreGradsC(*([FAKE] * 8))
    call = lambda c, dphi=FAKE, o=ctypes.byref(out), ws=FAKE, n=BIG: lib.mol_score_grad(  # noqa: E731
        ctypes.byref(c), dphi, o, ws, n, None)
    assert call(c, dphi=None) == mol.MOL_EINVAL
    assert call(c, o=None) == mol.MOL_EINVAL
    assert call(c, ws=None) == mol.MOL_EINVAL
    assert call(c, ws=FAKE + 64) == mol.MOL_EINVAL
    assert call(c, n=100) == mol.MOL_EWORKSPACE
    for field, value, status in (("W2", None, mol.MOL_EINVAL), ("H", 257, mol.MOL_EUNSUPPORTED), ("B", 0, mol.MOL_EINVAL),
                                 ("d", 1025, mol.MOL_EUNSUPPORTED), ("Pq", 33, mol.MOL_EUNSUPPORTED), ("dtype", 5, mol.MOL_EUNSUPPORTED)):
        bad = mol.MolProblemC.from_buffer_copy(c)
        setattr(bad, field, value)
        assert call(bad) == status, field


@pytest.mark.parametrize("B,N,Pq,Px,d,H", [(1, 1, 1, 1, 1, 1), (65535, 8388608, 8, 8, 64, 64), (1024, 1 << 20, 8, 8, 64, 64),
                                           (1, 8388608, 8, 4, 128, 128), (4096, 100003, 64, 1, 1024, 256), (65535, 17, 1, 64, 768, 256)])
def test_score_grad_workspace_is_bounded(B, N, Pq, Px, d, H):
    """The pairs' gradients are kept for a slab of items only."""
    out = ctypes.c_size_t(0)
    c = mol.MolProblemC(B, N, Pq, Px, d, H, mol.MOL_BF16, *([FAKE] * 8))
    assert mol.load().mol_workspace_size(ctypes.byref(c), mol.MOL_OP_SCORE_GRAD, 0, 0, 0, ctypes.byref(out)) == mol.MOL_OK
    assert out.value < (256 << 20) + 4 * B * Pq * (40 * d + 64 * 32 + 3 * Px) + 16 * N * Px * d + (1 << 30)


@pytest.mark.parametrize("B,N,Pq,Px,d,H", [(1, 1 << 28, 1, 1, 64, 256), (1, 1 << 27, 1, 1, 1024, 8), (1, 1 << 25, 1, 8, 256, 64),
                                           (2, 1 << 24, 1, 64, 8, 256), (3, 1 << 28, 2, 2, 16, 16), (65535, 1 << 20, 8, 8, 64, 64)])
@pytest.mark.parametrize("dtype", [mol.MOL_BF16, mol.MOL_F32])
def test_score_grad_workspace_does_not_grow_with_the_corpus(B, N, Pq, Px, d, H, dtype):
    """A few slabs' worth of buffers, and the sums of what the queries have, whatever the number of items."""
    out = ctypes.c_size_t(0)
    c = mol.MolProblemC(B, N, Pq, Px, d, H, dtype, *([FAKE] * 8))
    assert mol.load().mol_workspace_size(ctypes.byref(c), mol.MOL_OP_SCORE_GRAD, 0, 0, 0, ctypes.byref(out)) == mol.MOL_OK
    per_query = 4 * Pq * (d * 3 + 64) + 8 * Pq * Px
    assert out.value < (1 << 30) + B * per_query + 64 * H * Pq * Px * 4 * 256


def _tensor(**kw):
    t = mol.MolAdamwTensorC(100, *([FAKE] * 11), None, mol.MOL_F32, mol.MOL_BF16, mol.MOL_STATE_E4M3, 0.1, 0)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def _adamw(tensor=None, n=1, opt=None, **kw):
    a = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0, grad_scale=None, lr_ptr=None, step_ptr=None)
    a.update(kw)
    o = mol.MolAdamwC(*a.values())
    t = (mol.MolAdamwTensorC * 1)(tensor or _tensor(n=0))
    return mol.load().mol_adamw_step(ctypes.byref(o) if opt is None else None, t, n, None)


@pytest.mark.parametrize("bad", [
    dict(lr=-1.0), dict(lr=NAN), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=NAN), dict(eps=0.0),
    dict(eps=NAN), dict(step=0), dict(n=-1), dict(opt=0), dict(tensor=_tensor(n=-1)), dict(tensor=_tensor(n=1 << 35)),
    dict(tensor=_tensor(p=None)), dict(tensor=_tensor(g=None)), dict(tensor=_tensor(m_out=None)),
    dict(tensor=_tensor(v_scale=None)), dict(tensor=_tensor(weight_decay=-1.0)), dict(tensor=_tensor(weight_decay=NAN)),
])
def test_adamw_refuses(bad):
    assert _adamw(**bad) == mol.MOL_EINVAL


@pytest.mark.parametrize("bad", [dict(param_dtype=2), dict(grad_dtype=-1), dict(state=2)])
def test_adamw_refuses_types(bad):
    assert _adamw(tensor=_tensor(**bad)) == mol.MOL_EUNSUPPORTED


def test_adamw_of_nothing():
    assert _adamw(n=0) == mol.MOL_OK
    assert _adamw(tensor=_tensor(n=0, p=None)) == mol.MOL_OK
    mol.adamw_step(mol.AdamwTensors([], [], [], []))


# ---------------------------------------------------------------- what the binding sees
def test_binding_refuses_what_the_library_cannot_see():
    f, i32 = torch.zeros(2, 5, 8), torch.zeros(3, dtype=torch.int32)
    bad = [
        lambda: mol.embed_lookup(f, i32),                                       # not on a GPU
        lambda: mol.embed_lookup(f, i32.long()),                                # 64-bit ids
        lambda: mol.embed_lookup(f.half(), i32),
        lambda: mol.embed_lookup(f, i32, dtype=torch.float64),
        lambda: mol.embed_lookup(f[0], i32),
        lambda: mol.embed_lookup(f.transpose(1, 2), i32),
        lambda: mol.embed_grad(f, i32, 10),                                     # 5 rows, 3 ids
        lambda: mol.embed_grad(f, torch.zeros(5, dtype=torch.int32), 10, accumulate=True),
        lambda: mol.softmax_loss(f[0], i32[:2]),                                # 5 rows, 2 targets
        lambda: mol.softmax_loss(f[0].bfloat16(), torch.zeros(5, dtype=torch.int32)),
        lambda: mol.softmax_loss(f[0], torch.zeros(5)),
        lambda: mol.softmax_loss(f[0], torch.zeros(5, dtype=torch.int32), ids=i32),
        lambda: mol.AdamwTensors([f], [f], [f], []),
        lambda: mol.AdamwTensors([f], [f[:, :4]], [f], [f]),
        lambda: mol.AdamwTensors([f], [f], [f], [f.bfloat16()]),
        lambda: mol.AdamwTensors([f], [f], [f.to(torch.float8_e4m3fn)], [f.to(torch.float8_e4m3fn)]),
        lambda: mol.AdamwTensors([f], [f], [f], [f], out=dict(q=[f])),
        lambda: mol.AdamwTensors([f], [f], [f], [f], weight_decay=[0.1, 0.2]),
        lambda: mol.adamw_step(mol.AdamwTensors([f], [f], [f], [f]), grad_scale=0.5),
        lambda: mol.adamw_step(mol.AdamwTensors([f], [f], [f], [f])),           # not on a GPU
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was taken")


def test_score_grad_refuses_a_problem_of_other_sizes():
    B, N, Pq, Px, d, H = 3, 5, 2, 2, 8, 6
    good = dict(Q=torch.zeros(B, Pq, d), X=torch.zeros(Px, N, d), a_q=torch.zeros(B, Pq * Px), a_x=torch.zeros(N, Pq * Px),
                W1=torch.zeros(H, Pq * Px), b1=torch.zeros(H), W2=torch.zeros(Pq * Px, H), b2=torch.zeros(Pq * Px))
    dphi = torch.zeros(B, N)
    for name, t in (("X", torch.zeros(Px, N, d + 8)), ("a_q", torch.zeros(B, 3)), ("a_x", torch.zeros(N - 1, 4)),
                    ("b1", torch.zeros(H + 1)), ("W2", torch.zeros(4, H - 1)), ("b2", torch.zeros(3)),
                    ("a_x", torch.zeros(N, 4, dtype=torch.bfloat16)), ("W1", torch.zeros(H, 4, dtype=torch.bfloat16)),
                    ("b2", None)):
        prob = mol.Problem(**dict(good, **{name: t}))
        with pytest.raises(ValueError):
            mol.score_grad(prob, dphi)
    with pytest.raises(ValueError, match="not on a GPU"):
        mol.score_grad(mol.Problem(**good), dphi)


# ---------------------------------------------------------------- the compiled kernels
@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_no_mfma_result_read_early(tmp_path):
    sources = ["mol_score_grad.hip", "mol_score_grad_bf16.hip"]
    with cf.ThreadPoolExecutor() as ex:
        listings = dict(zip(sources, ex.map(lambda s: _asm(s, str(tmp_path)), sources)))
    bad = {s: early_reads(a, need=8) for s, a in listings.items()}
    assert not any(bad.values()), bad
