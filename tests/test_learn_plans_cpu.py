"""What plans and learners hold on to and refuse before anything is launched (CPU only)."""
import gc
import weakref

import pytest
import torch

from paper_2407_15462_amd import mol


def test_adamw_plan_keeps_its_tensors_when_the_lists_change():
    """The descriptors hold addresses: whatever the caller does to the lists afterwards, the tensors stay."""
    f = lambda: torch.zeros(300)  # noqa: E731
    e = lambda: torch.zeros(300, dtype=torch.uint8).view(torch.float8_e4m3fn)  # noqa: E731
    s = lambda: torch.zeros(2)  # noqa: E731
    lists = dict(p=[f()], g=[f()], m=[e()], v=[e()], m_scale=[s()], v_scale=[s()])
    out = dict(p=[f()], m=[e()], v=[e()], m_scale=[s()], v_scale=[s()], copy=[f().bfloat16()])
    held = {k: weakref.ref(x[0]) for k, x in lists.items()}
    held.update({"out " + k: weakref.ref(x[0]) for k, x in out.items()})
    address = {k: r().data_ptr() for k, r in held.items()}
    plan = mol.AdamwTensors(**lists, out=out)
    for x in lists.values():
        x[0] = None
    for x in out.values():
        x.clear()
    out.clear()
    gc.collect()
    gone = [k for k, r in held.items() if r() is None]
    assert not gone, f"freed under the plan: {gone}"
    assert all(r().data_ptr() == address[k] for k, r in held.items())
    del plan
    gc.collect()
    assert all(r() is None for r in held.values())


# ---------------------------------------------------------------- sizes that the C ABI has no room for
def meta(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="meta")


I32, LONG = torch.int32, (1 << 31) + 5
SIZES = [
    ("table of 2^31 + 5 rows", lambda: mol.embed_lookup(meta(1, LONG, 4), meta(3, dtype=I32))),
    ("2^31 + 5 ids", lambda: mol.embed_lookup(meta(1, 7, 4), meta(LONG, dtype=I32))),
    ("2^32 + 5 ids", lambda: mol.embed_lookup(meta(1, 7, 4), meta((1 << 32) + 5, dtype=I32))),
    ("rows of 2^32 + 8", lambda: mol.embed_lookup(meta(1, 7, (1 << 32) + 8), meta(3, dtype=I32))),
    ("2^32 + 1 tables", lambda: mol.embed_lookup(meta((1 << 32) + 1, 1, 1), meta(3, dtype=I32))),
    ("gradient onto 2^32 + 5 rows", lambda: mol.embed_grad(meta(1, 3, 4), meta(3, dtype=I32), (1 << 32) + 5)),
    ("gradient of 2^32 + 5 tokens", lambda: mol.embed_grad(meta(1, (1 << 32) + 5, 4), meta((1 << 32) + 5, dtype=I32), 7)),
    ("its workspace", lambda: mol.embed_grad_workspace(meta(1, 3, 4), (1 << 32) + 5)),
    ("loss of 2^32 + 5 columns", lambda: mol.softmax_loss(meta(1, (1 << 32) + 5), meta(1, dtype=I32))),
    ("its workspace, of 2^32 + 5 columns", lambda: mol.mol_softmax_loss_workspace(1, (1 << 32) + 5)),
    ("loss of 2^32 + 1 rows", lambda: mol.softmax_loss(meta((1 << 32) + 1, 3), meta((1 << 32) + 1, dtype=I32))),
    ("scores of 2^32 + 5 items", lambda: mol.score_grad(
        mol.Problem(meta(1, 1, 4), meta(1, (1 << 32) + 5, 4), meta(1, 1), meta((1 << 32) + 5, 1), meta(1, 1), meta(1), meta(1, 1), meta(1)),
        meta(1, (1 << 32) + 5))),
    ("step 2^32 + 1", lambda: mol.adamw_step(mol.AdamwTensors([torch.zeros(3)], [torch.zeros(3)], [torch.zeros(3)], [torch.zeros(3)]),
                                             step=(1 << 32) + 1)),
]


@pytest.mark.parametrize("what,call", SIZES, ids=[s[0] for s in SIZES])
def test_sizes_past_32_bits_are_refused(what, call):
    """They would be cut off to other sizes on their way into the library."""
    with pytest.raises(ValueError, match="2\\^31"):
        call()


# ---------------------------------------------------------------- rates that float32 does not hold
@pytest.mark.parametrize("bad", [dict(eps=1e-46), dict(eps=1e-40), dict(eps=1e39), dict(eps=float("inf")), dict(lr=1e39),
                                 dict(lr=float("inf")), dict(decay=float("inf"))])
def test_adamw_refuses_rates_outside_float32(bad):
    """The step is taken in float32: there eps = 1e-46 is 0, and parameters that have had no gradient become 0 / 0."""
    a = dict(lr=1e-3, eps=1e-8, decay=0.0)
    a.update(bad)
    opt = mol.MolAdamwC(a["lr"], 0.9, 0.999, a["eps"], 1, 0, None, None, None)
    t = (mol.MolAdamwTensorC * 1)(mol.MolAdamwTensorC(0, *([None] * 12), 0, 0, 0, a["decay"], 0))
    assert mol.load().mol_adamw_step(mol.ctypes.byref(opt), t, 1, None) == mol.MOL_EINVAL
    assert mol.load().mol_last_error()


@pytest.mark.parametrize("good", [dict(eps=1.2e-38), dict(eps=3e38), dict(lr=0.0), dict(lr=3e38)])
def test_adamw_takes_rates_of_float32(good):
    a = dict(lr=1e-3, eps=1e-8)
    a.update(good)
    opt = mol.MolAdamwC(a["lr"], 0.9, 0.999, a["eps"], 1, 0, None, None, None)
    t = (mol.MolAdamwTensorC * 1)(mol.MolAdamwTensorC(0, *([None] * 12), 0, 0, 0, 0.0, 0))
    assert mol.load().mol_adamw_step(mol.ctypes.byref(opt), t, 1, None) == mol.MOL_OK
