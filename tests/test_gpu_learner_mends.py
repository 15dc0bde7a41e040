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
