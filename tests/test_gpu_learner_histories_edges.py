"""The learner's steps with histories, norms and components of length one where
a row, a component or a history holds nothing (MI355X only)."""
import pytest
import torch

from test_gpu_learner_histories import batch, make, step64

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
