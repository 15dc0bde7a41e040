"""The learner's steps with histories, norms and components of length one where
a row, a component or a history holds nothing (MI355X only)."""
import pytest
import torch

import rows_helpers as rh
from test_gpu_learner_histories import OPTIONS, Rounded, batch, everything, make, step64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("options", [dict(normalize=True), dict(normalize=True, dropout=0.1), dict(normalize=True, states_8bit=True)])
def test_an_items_component_of_length_zero_has_no_gradient(options):
    """A padding or a new item: its zero components score 0, and what the loss wants of them has no direction."""
    Vq, V, Pq, Px, d, H, B, N = 20, 90, 4, 4, 64, 32, 9, 60
    learner = make(Vq, V, Pq, Px, d, H, seed=1, **options)
    zero = [(1, 7), (0, 7), (3, 50)]
    for p, row in zero:
        learner.master["items"][p, row] = 0
        learner.copy["items"][p, row] = 0
    ids, items, target, _ = batch(learner, B, N, seed=3)
    items[8:11] = torch.tensor([7, 50, 7])                # negatives of every query, or positives
    _, want, _, amp = step64(learner, (ids, items, target, None), 20.0)
    learner.step(ids.cuda(), items.cuda(), target.cuda(), 0.01)
    got = learner.grad["items"]
    live = torch.ones(Px, V, dtype=torch.bool)
    for p, row in zero:
        assert not got[p, row].any(), (p, row)
        live[p, row] = False
        assert not learner.master["items"][p, row].any(), (p, row)
    # the others' as ever: the bound of a step's gradients of items (softmax within 4e-3, scores within 1e-4, three roundings)
    got, want = got.double().cpu()[live], want["items"][live]
    assert torch.isfinite(want).all()
    assert float((got - want).norm() / want.norm()) < (4e-3 + 1e-4 + 3 * 2.0 ** -8) * amp
    if "states_8bit" in options:
        assert float(learner.state["m_scale"]["items"].max()) < 1.0 and float(learner.state["v_scale"]["items"].max()) < 1.0


def beta_of_queries_without_events(learner, ids, inv_temp):
    """What these queries' losses, of all queries' mean, are to beta, which is their row behind the norm: the gradient, and
    its size before normalize takes what lies along a component away."""
    q, items, target, offsets = ids
    Vq, V, Pq, Px, P, d = learner.shape
    inside = (q >= 0) & (q < Vq)
    dead = [b for b in range(len(target)) if not (inside[b] if offsets is None else inside[offsets[b]:offsets[b + 1]].any())]
    assert dead
    w = {n: learner.copy.get(n, t).double().cpu() for n, t in learner.master.items()}
    beta = w["beta"].requires_grad_()
    u = beta.view(Pq, d).expand(len(dead), Pq, d)
    r = u.norm(dim=-1, keepdim=True) if learner.normalize else torch.ones(1, dtype=torch.float64)
    Q = Rounded.apply(u / r)
    at = items.long().clamp(min=0)
    x = w["items"][:, at] * (items >= 0)[None, :, None]
    if learner.dropout:
        share = 1 - int(learner.dropout * 65536 + 0.5) / 65536
        x = Rounded.apply(x * rh.kept(x.numel(), learner.dropout, learner.seed, int(learner.steps), 1 << 40).view(x.shape) / share)
    X = Rounded.apply(x / x.norm(dim=-1, keepdim=True).clamp(min=1e-12)) if learner.normalize else x
    # (the gating logits are the last id's, where that is one of the table's: none of a query without an event is)
    s = torch.einsum("bqd,xnd->bnqx", Q, X).reshape(len(dead), len(items), P)
    lg = (w["a_x"][at] * (items >= 0)[:, None])[None] + torch.nn.functional.silu(s @ w["W1"].t() + w["b1"]) @ w["W2"].t() + w["b2"]
    hot = target[dead].long()
    keep = (items >= 0)[None] & (items[None] != items[hot][:, None])
    keep[torch.arange(len(dead)), hot] = True
    z = ((torch.softmax(lg, -1) * s).sum(-1) * inv_temp).masked_fill(~keep, -torch.inf)
    loss = (torch.logsumexp(z, 1) - z[torch.arange(len(dead)), hot]).sum() / len(target)
    gb, gq = torch.autograd.grad(loss, [beta, Q])
    return gb, float((gq.norm(dim=-1, keepdim=True) / r.detach()).sum(0).norm())


@pytest.mark.parametrize("name", ["norm", "gates norm", "all"])
@pytest.mark.parametrize("Vq,V,Pq,Px,d,H,B,N", [(50, 300, 8, 4, 64, 64, 40, 120), (20, 90, 4, 4, 24, 32, 9, 33)])
def test_beta_learns_from_queries_without_events(name, Vq, V, Pq, Px, d, H, B, N):
    """Behind the norm a query without an event is beta: its loss is one of the losses, so that a step's gradient of beta
    holds its part, and that of nothing else of a query's does."""
    learner = make(Vq, V, Pq, Px, d, H, seed=1, **OPTIONS[name])
    for step in range(1, 3):
        ids = batch(learner, B, N, seed=step)
        if ids[3] is None:
            ids[0][3], ids[0][6] = -1, Vq                  # (of queries without histories: ids outside the table)
        loss, want, amp_q, amp_x = step64(learner, ids, 20.0)          # (which takes these queries for constants)
        part, size = beta_of_queries_without_events(learner, ids, 20.0)
        assert float(part.norm()) > 0.1 * float(want["beta"].norm())
        got = learner.step(*(x.cuda() for x in ids[:3]), 0.01, offsets=None if ids[3] is None else ids[3].cuda())
        # the bounds of a step (scores within 1e-4, 20 times that in z, twice in the loss, once a component that falls to
        # the other side of its rounding; softmax within 4e-3 of itself, and the roundings on a gradient's way)
        assert float((got.double().cpu() - loss).abs().max()) < 4e-3 + 20 * 2.0 ** -8 / 24
        for n in learner.master:
            roundings = dict(queries=3, items=3, gates=4).get(n, 1)
            rel = 4e-3 + 1e-4 + roundings * 2.0 ** -8
            bound = rel * (amp_x if n == "items" else amp_q if roundings > 1 or n in ("gamma", "beta") else 1.0) * float(want[n].norm())
            if n == "beta":
                want[n], bound = want[n] + part, bound + rel * size
            assert float((learner.grad[n].double().cpu() - want[n]).norm()) < bound, n


def test_offsets_past_the_events_are_clamped_throughout():
    """As the scan clamps them: a history that starts behind the last event has no last event either."""
    a, b = (make(20, 90, 4, 4, 24, 32, seed=1, **OPTIONS["all"]) for _ in range(2))
    ids = (torch.arange(12, dtype=torch.int32) % 7).cuda()
    over, inside = (torch.tensor(o, dtype=torch.int32, device="cuda") for o in ([-3, 4, 9, 40, 50], [0, 4, 9, 12, 12]))
    _, items, target, _ = batch(a, 8, 40, seed=4)
    p, q = a.problem(ids, offsets=over), b.problem(ids, offsets=inside)
    assert all(torch.equal(x, y) for x, y in zip(p.tensors, q.tensors))
    assert not p.tensors[2][3].any(), "the gating logits of a history without events"
    losses = [m.step(ids, items.cuda(), target[:4].cuda(), 0.01, offsets=o) for m, o in ((a, over), (b, inside))]
    assert torch.equal(*losses)
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(everything(a), everything(b)))


def test_no_events_at_all():
    learner = make(20, 90, 4, 4, 24, 32, seed=1, **OPTIONS["all"])
    none, offsets = torch.empty(0, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    assert learner.states(none, offsets).shape == (3, 96) and not learner.states(none, offsets).any()
    kept = torch.rand(3, 96, device="cuda")
    assert torch.equal(learner.states(none, offsets, state=kept), kept)
    prob = learner.problem(none, offsets=offsets)
    unit = learner.master["beta"].view(4, 24)
    unit = unit / unit.norm(dim=-1, keepdim=True)
    # (one rounding to bfloat16, and float32's of the length)
    assert float((prob.tensors[0].float() - unit).abs().max()) < 2.0 ** -8 and not prob.tensors[2].any()
