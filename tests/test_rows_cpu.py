"""Refusals of the operators between embedding rows and scores: bad arguments are
turned down on the host, before anything is launched; and the oracle's generator (CPU only)."""
import ctypes

import numpy as np
import pytest
import torch

import rows_helpers as rh
from paper_2407_15462_amd import mol

FAKE, BIG = 256, 1 << 40          # a pointer that is never followed; every call below stops before its launch
NAN, INF = float("nan"), float("inf")
EINVAL, EUNSUPPORTED, EWORKSPACE = mol.MOL_EINVAL, mol.MOL_EUNSUPPORTED, mol.MOL_EWORKSPACE


def _call(name, defaults, bad):
    a = dict(defaults, **bad)
    return getattr(mol.load(), name)(*a.values(), None)


NORM = dict(x=FAKE, xt=0, T=5, d=8, gamma=None, beta=None, eps=1e-5, y=FAKE, yt=1)
NORM_GRAD = dict(dy=FAKE, dt=0, x=FAKE, xt=0, T=5000, d=8, gamma=None, eps=1e-5, dx=FAKE, ot=0, dgamma=FAKE, dbeta=FAKE, ws=FAKE,
                 n=BIG)
UNIT = dict(x=FAKE, xt=0, T=5, d=8, eps=1e-12, y=FAKE, yt=1)
UNIT_GRAD = dict(dy=FAKE, dt=0, x=FAKE, xt=0, T=5, d=8, eps=1e-12, dx=FAKE, ot=0)
DROP = dict(x=FAKE, xt=0, n=100, p=0.2, seed=1, offset=0, step=0, step_ptr=None, residual=None, y=FAKE, yt=1)
SCAN = dict(gate=FAKE, x=FAKE, xt=0, T=5000, d=8, offsets=FAKE, B=3, h0=None, h=FAKE, ht=1, last=None, ws=FAKE, n=BIG)
SCAN_GRAD = dict(gate=FAKE, x=FAKE, xt=0, h=FAKE, dh=FAKE, ht=1, T=5000, d=8, offsets=FAKE, B=3, h0=None, dlast=None, dgate=FAKE,
                 dx=FAKE, dh0=None, ws=FAKE, n=BIG)
STEP = dict(gate=FAKE, x=FAKE, xt=0, B=5, d=8, state=FAKE, out=FAKE, h=FAKE, ht=1)

ROWS = [(dict(T=-1), EINVAL), (dict(d=0), EINVAL), (dict(d=16385), EUNSUPPORTED), (dict(T=1 << 40), EUNSUPPORTED),
        (dict(eps=0.0), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=NAN), EINVAL), (dict(eps=INF), EINVAL), (dict(x=None), EINVAL),
        (dict(xt=2), EUNSUPPORTED)]
GRAD = [(dict(dy=None), EINVAL), (dict(dx=None), EINVAL), (dict(dt=3), EUNSUPPORTED), (dict(ot=-1), EUNSUPPORTED)]
TOKENS = [(dict(T=-1), EINVAL), (dict(d=0), EINVAL), (dict(B=0), EINVAL), (dict(d=65537), EUNSUPPORTED),
          (dict(T=(1 << 30) + 1), EUNSUPPORTED), (dict(B=(1 << 30) + 1), EUNSUPPORTED), (dict(T=1 << 30, d=65536), EUNSUPPORTED),
          (dict(xt=2), EUNSUPPORTED), (dict(ht=2), EUNSUPPORTED), (dict(gate=None), EINVAL), (dict(x=None), EINVAL),
          (dict(h=None), EINVAL), (dict(offsets=None), EINVAL), (dict(ws=None), EINVAL), (dict(ws=FAKE + 8), EINVAL),
          (dict(n=100), EWORKSPACE)]


@pytest.mark.parametrize("name,defaults,bad,status", [
    ("mol_layer_norm", NORM, b, s) for b, s in ROWS + [(dict(y=None), EINVAL), (dict(yt=7), EUNSUPPORTED)]] + [
    ("mol_layer_norm_grad", NORM_GRAD, b, s) for b, s in ROWS + GRAD + [
        (dict(dgamma=None), EINVAL), (dict(dbeta=None), EINVAL), (dict(ws=None), EINVAL), (dict(ws=FAKE + 4), EINVAL),
        (dict(n=64), EWORKSPACE)]] + [
    ("mol_normalize", UNIT, b, s) for b, s in ROWS + [(dict(y=None), EINVAL), (dict(yt=7), EUNSUPPORTED), (dict(eps=1.5), EINVAL)]] + [
    ("mol_normalize_grad", UNIT_GRAD, b, s) for b, s in ROWS + GRAD + [(dict(eps=2.0), EINVAL)]] + [
    ("mol_dropout", DROP, b, s) for b, s in [
        (dict(n=-1), EINVAL), (dict(n=1 << 40), EINVAL), (dict(p=-0.1), EINVAL), (dict(p=1.0), EINVAL), (dict(p=NAN), EINVAL),
        (dict(p=0.999999), EINVAL), (dict(offset=4), EINVAL), (dict(xt=2), EUNSUPPORTED), (dict(yt=2), EUNSUPPORTED),
        (dict(x=None), EINVAL), (dict(y=None), EINVAL)]] + [
    ("mol_gated_scan", SCAN, b, s) for b, s in TOKENS + [(dict(h0=FAKE, last=FAKE), EINVAL)]] + [
    ("mol_gated_scan_grad", SCAN_GRAD, b, s) for b, s in TOKENS + [
        (dict(dh=None), EINVAL), (dict(dgate=None), EINVAL), (dict(dx=None), EINVAL), (dict(dlast=FAKE, dh0=FAKE), EINVAL)]] + [
    ("mol_gated_step", STEP, b, s) for b, s in [
        (dict(B=-1), EINVAL), (dict(d=0), EINVAL), (dict(d=65537), EUNSUPPORTED), (dict(B=1 << 30), EUNSUPPORTED),
        (dict(xt=2), EUNSUPPORTED), (dict(ht=2), EUNSUPPORTED), (dict(gate=None), EINVAL), (dict(x=None), EINVAL),
        (dict(state=None), EINVAL), (dict(out=None), EINVAL)]])
def test_refuses(name, defaults, bad, status):
    assert _call(name, defaults, bad) == status
    assert mol.load().mol_last_error()


def test_nothing_to_do_needs_no_pointer():
    for name, defaults, none in (("mol_layer_norm", NORM, dict(T=0, x=None, y=None)), ("mol_normalize", UNIT, dict(T=0, x=None, y=None)),
                                 ("mol_normalize_grad", UNIT_GRAD, dict(T=0, x=None, dy=None, dx=None)),
                                 ("mol_layer_norm_grad", NORM_GRAD, dict(T=0, x=None, dy=None, dx=None, dgamma=None, dbeta=None)),
                                 ("mol_dropout", DROP, dict(n=0, x=None, y=None)),
                                 ("mol_gated_scan", SCAN, dict(T=0, gate=None, x=None, h=None, ws=None)),
                                 ("mol_gated_scan_grad", SCAN_GRAD, dict(T=0, gate=None, x=None, h=None, dgate=None, dx=None, ws=None)),
                                 ("mol_gated_step", STEP, dict(B=0, gate=None, x=None, state=None, out=None))):
        assert _call(name, defaults, none) == mol.MOL_OK, name


def test_workspaces_serve_smaller_calls():
    last = 0
    for T in list(range(0, 3000, 17)) + [10000, 1 << 20, 1 << 30]:
        n = mol.mol_layer_norm_grad_workspace(T, 640)
        assert n >= last
        last = n
    assert last <= 1024 * 2 * 640 * 4
    for T in (3, 500, 5000):
        sizes = [mol.mol_layer_norm_grad_workspace(T, d) for d in range(1, 16385, 13)]
        assert sizes == sorted(sizes)
        sizes = [mol.mol_gated_scan_workspace(T, d, 4) for d in range(1, 3000, 7)]
        assert sizes == sorted(sizes)
    sizes = [mol.mol_gated_scan_workspace(T, 96, 4) for T in range(0, 100000, 61)]
    assert sizes == sorted(sizes) and sizes[0] == 0
    # a small part of what a scan reads
    assert mol.mol_gated_scan_workspace(1 << 18, 512, 1000) < (1 << 18) * 512 * 4 // 8
    with pytest.raises(mol.MolError):
        mol.mol_gated_scan_workspace(5, 0, 1)
    assert mol.load().mol_gated_scan_workspace(1, 1, 1, None) == EINVAL
    assert mol.load().mol_layer_norm_grad_workspace(1, 1, None) == EINVAL


def test_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(4, 6)
    off = torch.zeros(3, dtype=torch.int32)
    for call, what in [
        (lambda: mol.layer_norm(x), "not on a GPU"), (lambda: mol.layer_norm(x.double()), "dtype"),
        (lambda: mol.layer_norm(x.t()), "contiguous"), (lambda: mol.layer_norm(x, gamma=torch.zeros(5)), "shape"),
        (lambda: mol.layer_norm_grad(x[:3], x), "shape"), (lambda: mol.normalize([1.0]), "tensor"),
        (lambda: mol.normalize(torch.zeros(3, 0)), "tensor"), (lambda: mol.normalize_grad(x.half(), x), "dtype"),
        (lambda: mol.dropout(x, 0.1, 1, step=-1), "step"), (lambda: mol.dropout(x, 0.1, 1, step=1 << 32), "step"),
        (lambda: mol.dropout(x, 0.1, 1, offset=-8), "offset"), (lambda: mol.dropout(x, 0.1, 1, step=torch.zeros(2)), "one element"),
        (lambda: mol.dropout(x, 0.1, 1, residual=x[0]), "shape"), (lambda: mol.gated_scan(x, x[0]), "tensor"),
        (lambda: mol.gated_scan(x.bfloat16(), x), "dtype"), (lambda: mol.gated_scan(x, x, offsets=off.long()), "dtype"),
        (lambda: mol.gated_scan(x, x, offsets=off[:1]), "offsets"), (lambda: mol.gated_scan(x, x, offsets=off, h0=x), "shape"),
        (lambda: mol.gated_scan_grad(x, x, x, dh=x.bfloat16()), "dtype"), (lambda: mol.gated_scan_grad(x, x, x[:2], dh=x), "shape"),
        (lambda: mol.gated_scan_grad(x, x, x, dlast=x), "shape"), (lambda: mol.gated_step(x, x, x.bfloat16()), "dtype"),
        (lambda: mol.gated_step(x, x, x[:2]), "shape"), (lambda: mol.gated_step(x, x, x), "not on a GPU"),
    ]:
        with pytest.raises(ValueError, match=what):
            call()


def test_the_oracles_generator_gives_the_published_answers():
    c = np.array([[0, 0, 0, 0], [0xFFFFFFFF] * 4, [0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344]], dtype=np.uint64)
    for counter, key, want in ((c[0], (0, 0), "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
                               (c[1], (0xFFFFFFFF, 0xFFFFFFFF), "408f276d 41c83b0e a20bc7c6 6d5451fd"),
                               (c[2], (0xA4093822, 0x299F31D0), "d16cfe09 94fdcceb 5001e420 24126ea1")):
        assert " ".join(f"{v:08x}" for v in rh.philox(counter, key)) == want
    share = float(rh.kept(1 << 20, 0.3, 7, 1, 0).double().mean())
    assert abs(share - 0.7) < 5 * (0.21 / (1 << 20)) ** 0.5


def test_workspace_query_writes_whole_size():
    out = ctypes.c_size_t(0)
    assert mol.load().mol_gated_scan_workspace(1 << 23, 8192, 1, ctypes.byref(out)) == mol.MOL_OK
    assert out.value > 1 << 32
