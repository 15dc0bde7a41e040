"""The operators that learn the similarity, together: lookup, scores, loss,
gradients and AdamW in one step, against the same step in float64, captured
into a graph, and the retrieval that follows it (MI355X only)."""
import pytest
import torch

from oracle import mol_oracle as mo
from paper_2407_15462_amd import mol
from parity_helpers import check_topk_row, log

pytestmark = pytest.mark.gpu

NAMES = ("queries", "items", "a_q", "a_x", "W1", "b1", "W2", "b2")


def make(Vq, V, Pq, Px, d, H, seed, **kw):
    gen = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    unit = lambda v: v / v.norm(dim=-1, keepdim=True)  # noqa: E731
    P = Pq * Px
    t = dict(queries=unit(randn(Vq, Pq, d)), items=unit(randn(Px, V, d)), a_q=0.1 * randn(Vq, P), a_x=0.1 * randn(V, P),
             W1=0.1 * randn(H, P), b1=0.1 * randn(H), W2=0.1 * randn(P, H), b2=0.1 * randn(P))
    return mol.Learner(*(t[n].cuda().contiguous() for n in NAMES), **kw), t


def batch(Vq, V, B, N, seed):
    gen = torch.Generator().manual_seed(seed)
    q = torch.randint(0, Vq, (B,), generator=gen).int()
    items = torch.randint(0, V, (N,), generator=gen).int()
    items[5] = -1                                        # an empty slot
    target = torch.randint(6, N, (B,), generator=gen).int()
    items[7] = items[target[0]]                          # a copy of a positive
    return q, items, target


def step64(p, copies, state, ids, lr, inv_temp, decay, step):
    """One step in float64 on masters p, scoring with the bfloat16 copies: losses and gradients, p and state updated."""
    q, items, target = (t.long() for t in ids)
    w = {n: (copies[n] if n in copies else p[n]).double().clone().requires_grad_() for n in NAMES}
    ok = items >= 0
    it = items.clamp(min=0)
    Q, X = w["queries"][q], w["items"][:, it] * ok[None, :, None]
    aq, ax = w["a_q"][q], w["a_x"][it] * ok[:, None]
    B, N = len(q), len(items)
    s = torch.einsum("bqd,xnd->bnqx", Q, X).reshape(B, N, -1)
    lg = aq[:, None] + ax[None] + torch.nn.functional.silu(s @ w["W1"].t() + w["b1"]) @ w["W2"].t() + w["b2"]
    phi = (torch.softmax(lg, -1) * s).sum(-1)
    keep = ok[None] & (items[None] != items[target][:, None])
    keep[torch.arange(B), target] = True
    z = (phi * inv_temp).masked_fill(~keep, -torch.inf)
    loss = torch.logsumexp(z, 1) - z[torch.arange(B), target]
    g = dict(zip(NAMES, torch.autograd.grad(loss.mean(), [w[n] for n in NAMES])))
    for n in NAMES:
        m, v = state[n]
        m += 0.1 * (g[n] - m)
        v += 0.001 * (g[n] * g[n] - v)
        hat = (m / (1 - 0.9 ** step)) / ((v / (1 - 0.999 ** step)).sqrt() + 1e-8)
        p[n] = p[n] - lr * (hat + (decay if n in copies else 0.0) * p[n])
    return loss.detach(), g


@pytest.mark.parametrize("states_8bit", [False, True])
@pytest.mark.parametrize("Vq,V,Pq,Px,d,H,B,N", [(50, 300, 8, 4, 64, 64, 40, 120), (20, 90, 4, 4, 24, 32, 9, 33)])
def test_step_follows_float64(Vq, V, Pq, Px, d, H, B, N, states_8bit):
    log(f"[learner] Vq={Vq} V={V} {Pq}x{Px} d={d} H={H} B={B} N={N} 8-bit states: {states_8bit}")
    learner, t = make(Vq, V, Pq, Px, d, H, seed=1, weight_decay=0.01, states_8bit=states_8bit)
    lr = torch.tensor([0.01], device="cuda")
    for step in range(1, 4):
        ids = batch(Vq, V, B, N, seed=step)
        # the step's reference starts from where the learner is
        p = {n: learner.master[n].double().cpu() for n in NAMES}
        copies = {n: learner.copy[n].cpu() for n in learner.copy}
        assert all(torch.equal(copies[n], p[n].to(torch.float32).bfloat16()) for n in copies), "the copies are behind"
        state = {n: tuple(value(learner, k, n) for k in ("m", "v")) for n in NAMES}
        loss, g = step64(p, copies, state, ids, 0.01, 20.0, 0.01, step)
        got = learner.step(*(x.cuda() for x in ids), lr)
        assert int(learner.steps) == step
        # scores are within 1e-4 (the library's stated precision), so that z and the
        # loss are within 20 times that, twice
        assert float((got.double().cpu() - loss).abs().max()) < 4e-3
        for n in NAMES:
            # softmax within 4e-3 of itself, one bf16 rounding of the row gradients and of dW
            rel = float((learner.grad[n].double().cpu() - g[n]).norm() / g[n].norm())
            assert rel < 4e-3 + 2.0 ** -8 + 1e-4, (n, rel)
            # at most lr times (1 / bias of the first steps) an element, and nothing where there is no gradient
            moved = (learner.master[n].double().cpu() - p[n]).abs()
            still = (g[n] == 0) & (state[n][0].abs() < 1e-12)
            assert float(moved[still].max() if bool(still.any()) else 0.0) < 1e-6, n
            assert float(moved.norm() / (0.01 * moved.numel() ** 0.5)) < 0.1, n


def value(learner, k, n):
    """A state of a tensor in float64 (8-bit states: the values that they stand for, v squared)."""
    x = learner.state[k][n]
    if x.dtype != torch.float8_e4m3fn:
        return x.double().cpu()
    i = NAMES.index(n)
    s = learner.tensors.tensors[4 if k == "m" else 5][i].double().cpu()
    y = x.float().double().cpu().flatten() * s.repeat_interleave(256)[:x.numel()]
    return (y if k == "m" else y * y).view(x.shape)


def test_captured_step_replays_as_eager_ones():
    """A step captured once and replayed, with eager work and other inputs between the replays: the bits of eager steps."""
    Vq, V, B, N = 40, 200, 16, 64
    eager, _ = make(Vq, V, 8, 8, 32, 64, seed=3, states_8bit=True)
    learner, _ = make(Vq, V, 8, 8, 32, 64, seed=3, states_8bit=True)
    batches = [tuple(x.cuda() for x in batch(Vq, V, B, N, seed=10 + k)) for k in range(5)]
    held = [x.clone() for x in batches[0]]
    lr = torch.tensor([0.01], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = learner.step(*held, lr)                  # warm-up, and step 1
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(first, eager.step(*batches[0], lr))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = learner.step(*held, lr)
    for k in range(1, 5):
        for h, x in zip(held, batches[k]):
            h.copy_(x)
        loss.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = eager.step(*batches[k], lr)
        assert torch.equal(loss, want), f"replay {k}"
        assert int(learner.steps) == k + 1
        for n in NAMES:
            assert torch.equal(learner.master[n], eager.master[n]), (k, n)


def test_two_streams_at_once():
    """Two models trained on two streams without waiting: each as alone."""
    Vq, V, B, N = 60, 400, 32, 96
    ids = tuple(x.cuda() for x in batch(Vq, V, B, N, seed=2))
    lr = torch.tensor([0.01], device="cuda")
    alone = [make(Vq, V, 4, 4, 64, 32, seed=s)[0] for s in (5, 6)]
    both = [make(Vq, V, 4, 4, 64, 32, seed=s)[0] for s in (5, 6)]
    for m in alone:
        for _ in range(4):
            m.step(*ids, lr)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        for m, s in zip(both, streams):
            with torch.cuda.stream(s):
                m.step(*ids, lr)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        assert all(torch.equal(a.master[n], b.master[n]) for n in NAMES)


def test_retrieval_with_the_trained_model():
    """The items' copy is the corpus: exact top-k of the model after its steps equals the oracle's."""
    Vq, V, k = 30, 500, 20
    learner, _ = make(Vq, V, 8, 4, 64, 64, seed=4, weight_decay=0.01)
    lr = torch.tensor([0.003], device="cuda")
    for step in range(3):
        learner.step(*(x.cuda() for x in batch(Vq, V, 24, 100, seed=20 + step)), lr)
    prob = learner.problem(torch.arange(12, dtype=torch.int32, device="cuda"))
    s, i = mol.topk_exact(prob, k)
    names = ("Q", "X", "a_q", "a_x", "W1", "b1", "W2", "b2")
    arrays = {n: (t.cpu().view(torch.int16).numpy().view("u2") if t.dtype == torch.bfloat16 else t.cpu().numpy())
              for n, t in zip(names, prob.tensors)}
    phi = mo.mol_scores(mo.Problem.from_arrays(dict(arrays, dtype="bf16")), list(range(12)))
    for b in range(12):
        check_topk_row(phi[b], i[b].cpu().numpy(), s[b].cpu().numpy(), k, f"trained query {b}")
