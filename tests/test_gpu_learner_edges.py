"""A learner's saved state, ids past its tables, the gating's precision and
refusals that leave it as it was (MI355X only)."""
import pytest
import torch

from paper_2407_15462_amd import mol
from parity_helpers import log
from test_gpu_learner import NAMES, batch, make, step64

pytestmark = pytest.mark.gpu


def bits(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def same(a, b):
    return all(torch.equal(a.master[n], b.master[n]) for n in NAMES) and \
        all(torch.equal(bits(a.state[k][n]), bits(b.state[k][n])) for k in a.state for n in a.state[k])


@pytest.mark.parametrize("states_8bit", [False, True])
def test_a_saved_learner_goes_on_bit_for_bit(states_8bit):
    """master, state and steps are all of a learner: 3 steps, saved and loaded, and 3 more are 6 steps."""
    Vq, V, B, N = 40, 300, 16, 64
    whole, _ = make(Vq, V, 8, 4, 32, 32, seed=3, states_8bit=states_8bit, weight_decay=0.01)
    ids = [tuple(x.cuda() for x in batch(Vq, V, B, N, seed=30 + k)) for k in range(6)]
    lr = torch.tensor([0.01], device="cuda")
    for k in range(3):
        whole.step(*ids[k], lr)
    saved = {n: t.clone() for n, t in whole.master.items()}
    state = {k: {n: t.clone() for n, t in d.items()} for k, d in whole.state.items()}
    again = mol.Learner(*(saved[n] for n in NAMES), weight_decay=0.01, states_8bit=states_8bit)
    for k, d in state.items():
        for n, t in d.items():
            again.state[k][n].copy_(t)
    again.steps.copy_(whole.steps)
    assert same(whole, again)
    for k in range(3, 6):
        assert torch.equal(whole.step(*ids[k], lr), again.step(*ids[k], lr)), k
    assert same(whole, again)
    assert ("m_scale" in whole.state) == ("v_scale" in whole.state) == states_8bit


def test_an_item_id_past_the_table_is_an_empty_slot():
    """In all of a step, as in the lookup: not a negative of score 0, and no positive."""
    Vq, V, B, N = 40, 200, 16, 64
    lr = torch.tensor([0.01], device="cuda")
    q, items, target = (x.cuda() for x in batch(Vq, V, B, N, seed=1))
    target[3] = 9
    got = []
    for empty in (-1, V, 2 ** 31 - 1):
        learner, _ = make(Vq, V, 4, 4, 32, 32, seed=2)
        ids = items.clone()
        ids[9] = ids[40] = empty                          # a positive among them, and a negative
        got.append((learner.step(q, ids, target, lr), learner))
        assert float(got[-1][0][3]) == 0.0, "the positive of query 3 is an empty slot"
        assert ids[9] == empty, "the caller's ids were written"
    for loss, learner in got[1:]:
        assert torch.equal(loss, got[0][0]) and same(learner, got[0][1])


def test_a_query_id_past_the_table_adds_to_no_gradient():
    Vq, V, B, N = 40, 200, 16, 64
    lr = torch.tensor([0.01], device="cuda")
    q, items, target = (x.cuda() for x in batch(Vq, V, B, N, seed=1))
    learners = []
    for empty, at in ((-1, 11), (Vq, 11), (-1, 20)):      # (whatever its positive is)
        learner, _ = make(Vq, V, 4, 4, 32, 32, seed=2)
        ids, t = q.clone(), target.clone()
        ids[2], t[2] = empty, at
        loss = learner.step(ids, items, t, lr)
        assert bool(torch.isfinite(loss).all())
        learners.append(learner)
    assert same(learners[0], learners[1]) and same(learners[0], learners[2])


# ---------------------------------------------------------------- refusals
def everything(learner):
    return [bits(t).clone() for d in (learner.master, learner.copy, learner.grad, *learner.state.values()) for t in d.values()] + \
        [learner.steps.clone()]


@pytest.mark.parametrize("bad", [dict(lr=-0.01), dict(lr=float("nan")), dict(lr=float("inf")), dict(lr=1e39), dict(lr=None),
                                 dict(lr="0.1"), dict(inv_temp=0.0), dict(inv_temp=float("inf")), dict(target="short"),
                                 dict(target="wide"), dict(items="wide"), dict(items="none"), dict(queries="none")])
def test_a_refused_step_changes_nothing(bad):
    Vq, V, B, N = 40, 200, 16, 64
    learner, _ = make(Vq, V, 4, 4, 32, 32, seed=2)
    q, items, target = (x.cuda() for x in batch(Vq, V, B, N, seed=1))
    learner.step(q, items, target, 0.01)
    before = everything(learner)
    kw = dict(lr=0.01, inv_temp=20.0)
    kw.update({k: x for k, x in bad.items() if k in kw})
    if "target" in bad:
        target = target[:-1] if bad["target"] == "short" else target.long()
    if "items" in bad:
        items = items.long() if bad["items"] == "wide" else items[:0]
    if bad.get("queries") == "none":
        q, target = q[:0], target[:0]
    with pytest.raises((ValueError, mol.MolError)):
        learner.step(q, items, target, **kw)
    assert all(torch.equal(a, b) for a, b in zip(before, everything(learner)))


# ---------------------------------------------------------------- precision of the gating MLP
@pytest.mark.parametrize("std", [0.5, 2.0])
@pytest.mark.parametrize("Vq,V,Pq,Px,d,H,B,N", [(50, 300, 8, 8, 64, 64, 40, 120), (20, 90, 4, 4, 24, 32, 9, 33)])
def test_a_step_with_large_gating_weights_follows_float64(Vq, V, Pq, Px, d, H, B, N, std):
    """Weights that have left the range of the float16 chain (RMS 0.3): the losses and gradients keep the precision of small ones."""
    log(f"[learner] Vq={Vq} V={V} {Pq}x{Px} d={d} H={H} B={B} N={N} weights of {std}")
    _, t = make(Vq, V, Pq, Px, d, H, seed=1)
    t["W1"], t["W2"] = t["W1"] * (std / 0.1), t["W2"] * (std / 0.1)
    learner = mol.Learner(*(t[n].cuda().contiguous() for n in NAMES))
    p = {n: learner.master[n].double().cpu() for n in NAMES}
    copies = {n: learner.copy[n].cpu() for n in learner.copy}
    state = {n: (torch.zeros_like(p[n]), torch.zeros_like(p[n])) for n in NAMES}
    ids = batch(Vq, V, B, N, seed=1)
    loss, g = step64(p, copies, state, ids, 0.01, 20.0, 0.0, 1)
    got = learner.step(*(x.cuda() for x in ids), 0.01)
    # scores within 1e-4 (the library's stated precision), z and the loss 20 times that, twice
    assert float((got.double().cpu() - loss).abs().max()) < 4e-3
    for n in NAMES:
        rel = float((learner.grad[n].double().cpu() - g[n]).norm() / g[n].norm())
        assert rel < 4e-3 + 2.0 ** -8 + 1e-4, (n, rel)


def test_the_gating_of_a_step_is_the_callers_choice():
    ids = tuple(x.cuda() for x in batch(50, 300, 40, 120, seed=4))
    losses, grads = {}, {}
    for name, kw in (("default", {}), ("f32", dict(flags=mol.MOL_FLAG_F32_GATING)), ("f16", dict(flags=0)),
                     ("all f32", dict(grad_flags=mol.MOL_FLAG_F32_GATING))):
        learner, _ = make(50, 300, 8, 8, 64, 64, seed=6, **kw)
        losses[name] = learner.step(*ids, 0.01)
        grads[name] = learner.grad["W1"].clone()
    assert torch.equal(losses["default"], losses["f32"]) and torch.equal(losses["default"], losses["all f32"])
    assert not torch.equal(losses["default"], losses["f16"]) and not torch.equal(grads["default"], grads["all f32"])
    # both gradients a rounding to bf16 away from the same values, and those float32's errors apart
    assert float((grads["default"] - grads["all f32"]).float().norm() / grads["default"].float().norm()) < 2.0 ** -8
    with pytest.raises(mol.MolError):
        make(50, 300, 8, 8, 64, 64, seed=6, flags=4)[0].step(*ids, 0.01)
