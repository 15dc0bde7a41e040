"""The learner with queries formed from histories, layer norm, components of length
one and dropout: the operators between embedding rows and scores together, in
a step against the same step in float64, captured into a graph, and in retrieval
from states that go on (MI355X only)."""
import pytest
import torch

import rows_helpers as rh
from oracle import mol_oracle as mo
from paper_2407_15462_amd import mol
from parity_helpers import check_topk_row, log

pytestmark = pytest.mark.gpu

NAMES = ("queries", "items", "a_q", "a_x", "W1", "b1", "W2", "b2")
OPTIONS = {
    "unit": dict(normalize=True), "norm": dict(norm=True), "drop": dict(dropout=0.25), "gates": dict(gates=True),
    "unit drop": dict(normalize=True, dropout=0.1), "all": dict(normalize=True, dropout=0.2, gates=True, norm=True),
    "gates norm": dict(gates=True, norm=True),
}


def make(Vq, V, Pq, Px, d, H, seed, gates=False, norm=False, **kw):
    gen = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    P = Pq * Px
    # (rows of about length one; the scores of unnormalised ones stay small)
    t = dict(queries=randn(Vq, Pq, d) / d ** 0.5, items=randn(Px, V, d) / d ** 0.5, a_q=0.1 * randn(Vq, P), a_x=0.1 * randn(V, P),
             W1=0.1 * randn(H, P), b1=0.1 * randn(H), W2=0.1 * randn(P, H), b2=0.1 * randn(P))
    if gates:
        kw["gates"] = (1 + randn(Vq, Pq, d)).cuda()
    if norm:
        kw["norm"] = ((1 + 0.2 * randn(Pq * d)).cuda() / d ** 0.5, (0.1 * randn(Pq * d) / d ** 0.5).cuda())
    return mol.Learner(*(t[n].cuda().contiguous() for n in NAMES), seed=77, **kw)


def batch(learner, B, N, seed):
    """(ids of queries or events, items, targets, offsets or None)"""
    Vq, V = learner.shape[:2]
    gen = torch.Generator().manual_seed(seed)
    items = torch.randint(0, V, (N,), generator=gen).int()
    items[5] = -1                                        # an empty slot
    target = torch.randint(6, N, (B,), generator=gen).int()
    if "gates" not in learner.master:
        return torch.randint(0, Vq, (B,), generator=gen).int(), items, target, None
    lens = torch.randint(0, 30, (B,), generator=gen)
    lens[1], lens[2] = 0, 1
    offsets = torch.cat([torch.tensor([2]), 2 + lens.cumsum(0)]).int()       # two events in front are no history's
    ids = torch.randint(0, Vq, (int(offsets[-1]) + 3,), generator=gen).int()
    ids[4], ids[int(offsets[4])] = -1, Vq                # events outside the table
    return ids, items, target, offsets


class Rounded(torch.autograd.Function):
    """To bfloat16 and back; the gradient as it is."""

    @staticmethod
    def forward(ctx, x):
        return x.bfloat16().double()

    @staticmethod
    def backward(ctx, g):
        return g


def step64(learner, ids, inv_temp):
    """Losses, gradients, and how much the gradients shrink on their way back through the norms."""
    q, items, target = (x.long() for x in ids[:3])
    offsets = ids[3]
    Vq, V, Pq, Px, P, d = learner.shape
    w = {n: learner.copy.get(n, t).double().cpu().requires_grad_() for n, t in learner.master.items()}
    steps, p = int(learner.steps), learner.dropout
    kept_share = 1 - int(p * 65536 + 0.5) / 65536

    def drop(x, offset):
        return x if not p else Rounded.apply(x * rh.kept(x.numel(), p, learner.seed, steps, offset).view(x.shape) / kept_share)

    inside = (q >= 0) & (q < Vq)
    rows = drop(w["queries"].reshape(Vq, Pq * d)[q.clamp(0, Vq - 1)] * inside[:, None], 0)
    if offsets is None:
        v, of_query = rows, q
    else:
        g = w["gates"].reshape(Vq, Pq * d)[q.clamp(0, Vq - 1)]
        f = torch.where(inside[:, None], torch.sigmoid(g), 1.0)
        states, of_query = [], []
        for a, b in zip(offsets[:-1].tolist(), offsets[1:].tolist()):
            s = torch.zeros(Pq * d, dtype=torch.float64)
            for t in range(a, b):
                s = f[t] * s + (1 - f[t]) * rows[t]
            states.append(s)
            of_query.append(int(q[b - 1]) if b > a else -1)
        v, of_query = torch.stack(states), torch.tensor(of_query)
    kept = [v]
    if "gamma" in w:
        c = v - v.mean(1, keepdim=True)
        v = c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt() * w["gamma"] + w["beta"]
        kept.append(v)
    Q = v.view(-1, Pq, d)
    if learner.normalize:
        Q = Q / Q.norm(dim=-1, keepdim=True).clamp(min=1e-12)
    kept.append(Q)
    Q = Rounded.apply(Q)
    if "gamma" in w:                                     # a query without an event adds to no gradient of a query's
        dead = ~inside if offsets is None else torch.tensor([not bool(inside[a:b].any()) for a, b in
                                                             zip(offsets[:-1].tolist(), offsets[1:].tolist())])
        Q = torch.where(dead[:, None, None], Q.detach(), Q)
    it = items.clamp(min=0)
    x = drop(w["items"][:, it] * (items >= 0)[None, :, None], 1 << 40)
    X = Rounded.apply(x / x.norm(dim=-1, keepdim=True).clamp(min=1e-12)) if learner.normalize else x
    aq = w["a_q"][of_query.clamp(0, Vq - 1)] * ((of_query >= 0) & (of_query < Vq))[:, None]
    ax = w["a_x"][it] * (items >= 0)[:, None]
    B, N = len(target), len(items)
    s = torch.einsum("bqd,xnd->bnqx", Q, X).reshape(B, N, -1)
    lg = aq[:, None] + ax[None] + torch.nn.functional.silu(s @ w["W1"].t() + w["b1"]) @ w["W2"].t() + w["b2"]
    phi = (torch.softmax(lg, -1) * s).sum(-1)
    keep = (items >= 0)[None] & (items[None] != items[target][:, None])
    keep[torch.arange(B), target] = True
    z = (phi * inv_temp).masked_fill(~keep, -torch.inf)
    loss = torch.logsumexp(z, 1) - z[torch.arange(B), target]
    names = list(w)
    got = torch.autograd.grad(loss.mean(), [w[n] for n in names] + kept + [x, X])
    g = dict(zip(names, got))
    back = got[len(names):]
    # a relative error of a norm's dy is one of its dx times |dy| / |dx|, dx taken to dy's scale (the gradient less
    # what lies along the row)
    size = lambda t: float(t.norm())  # noqa: E731
    amp_q = amp_x = 1.0
    if learner.normalize:
        before = kept[-2].view(-1, Pq, d)
        r = before.detach().norm(dim=-1, keepdim=True).clamp(min=1e-12)
        amp_q *= size(back[len(kept) - 1]) / size(back[len(kept) - 2].view(-1, Pq, d) * r)
        amp_x = size(back[-1]) / size(back[-2] * x.detach().norm(dim=-1, keepdim=True).clamp(min=1e-12))
    if "gamma" in w:
        v0 = kept[0].detach()
        std = ((v0 - v0.mean(1, keepdim=True)).square().mean(1, keepdim=True) + 1e-5).sqrt()
        amp_q *= size(back[1] * w["gamma"].detach()) / size(back[0] * std)
    return loss.detach(), g, max(amp_q, 1.0), max(amp_x, 1.0)


@pytest.mark.parametrize("name", OPTIONS)
@pytest.mark.parametrize("Vq,V,Pq,Px,d,H,B,N", [(50, 300, 8, 4, 64, 64, 40, 120), (20, 90, 4, 4, 24, 32, 9, 33)])
def test_step_follows_float64(name, Vq, V, Pq, Px, d, H, B, N):
    log(f"[learner] {name}: Vq={Vq} V={V} {Pq}x{Px} d={d} H={H} B={B} N={N}")
    learner = make(Vq, V, Pq, Px, d, H, seed=1, **OPTIONS[name])
    for step in range(1, 3):
        ids = batch(learner, B, N, seed=step)
        loss, g, amp_q, amp_x = step64(learner, ids, 20.0)
        before = {n: t.clone() for n, t in learner.master.items()}
        got = learner.step(*(x.cuda() for x in ids[:3]), 0.01, offsets=None if ids[3] is None else ids[3].cuda())
        assert int(learner.steps) == step
        # scores within 1e-4, 20 times that in z, twice in the loss; and a component next to a border of its rounding to
        # bfloat16 may fall to its other side, 2^-8 of one of d >= 24 terms of a score: 20 times 2^-8 / 24, once
        assert float((got.double().cpu() - loss).abs().max()) < 4e-3 + 20 * 2.0 ** -8 / 24
        half = 2.0 ** -8
        for n in learner.master:
            # softmax within 4e-3 of itself; roundings of dQ or dX, of dx or dgate and of the dropped gradient, of h in dgate
            roundings = dict(queries=3, items=3, gates=4, gamma=1, beta=1).get(n, 1)
            bound = (4e-3 + 1e-4 + roundings * half) * (amp_x if n == "items" else amp_q if roundings > 1 or n == "gamma" else 1.0)
            rel = float((learner.grad[n].double().cpu() - g[n]).norm() / g[n].norm())
            assert rel < bound, (n, rel, bound, amp_q, amp_x)
            assert not torch.equal(learner.master[n], before[n]), n


def everything(learner):
    return list(learner.master.values()) + [t for k in learner.state.values() for t in k.values()]


def test_captured_step_replays_as_eager_ones():
    """Dropout counts on with the replays, and the histories change under the graph."""
    B, N = 16, 64
    eager, learner = (make(40, 200, 8, 8, 32, 64, seed=3, states_8bit=True, **OPTIONS["all"]) for _ in range(2))
    batches = [[x.cuda() for x in batch(learner, B, N, seed=10 + k)] for k in range(5)]
    longest = max(len(b[0]) for b in batches)
    for b in batches:                                     # (events behind the last history are no history's)
        b[0] = torch.cat([b[0], torch.full((longest - len(b[0]),), 3, dtype=torch.int32, device="cuda")])
    held = [x.clone() for x in batches[0]]
    lr = torch.tensor([0.01], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = learner.step(*held[:3], lr, offsets=held[3])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(first, eager.step(*batches[0][:3], lr, offsets=batches[0][3]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = learner.step(*held[:3], lr, offsets=held[3])
    for k in range(1, 5):
        for h, x in zip(held, batches[k]):
            h.copy_(x)
        loss.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, eager.step(*batches[k][:3], lr, offsets=batches[k][3])), f"replay {k}"
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(everything(learner), everything(eager))), k


def test_states_that_go_on():
    """Histories in one scan, and as a prefill and single events: the same states up to a bfloat16 gate's and row's arithmetic."""
    learner = make(60, 300, 8, 4, 64, 64, seed=5, **OPTIONS["all"])
    gen = torch.Generator().manual_seed(1)
    ids = torch.randint(0, 60, (6, 25), generator=gen).int().cuda()
    ids[2, 20] = -1
    offsets = lambda n: (torch.arange(7, dtype=torch.int32) * n).cuda()  # noqa: E731
    want = learner.states(ids.reshape(-1), offsets(25))
    state = learner.states(ids[:, :10].reshape(-1).contiguous(), offsets(10))
    state = learner.states(ids[:, 10:18].reshape(-1).contiguous(), offsets(8), state=state)
    for t in range(18, 25):
        kept = state.clone()
        assert learner.advance(state, ids[:, t].contiguous()) is state
        assert not torch.equal(state, kept)
        assert t != 20 or torch.equal(state[2], kept[2]), "an event outside the table changes nothing"
    # 25 tokens, STEP and JOIN roundings each at most, of states of at most the largest row element
    assert float((state - want).abs().max()) < (rh.STEP * 25 + 3 * rh.JOIN) * rh.U * float(learner.copy["queries"].float().abs().max())
    a, b = learner.problem(ids.reshape(-1), offsets=offsets(25)), learner.problem_of(want, ids[:, 24].contiguous())
    assert all(torch.equal(x, y) for x, y in zip(a.tensors, b.tensors))


@pytest.mark.parametrize("name", ["unit", "all"])
def test_retrieval_with_the_trained_model(name):
    k = 20
    learner = make(30, 500, 8, 4, 64, 64, seed=4, weight_decay=0.01, **OPTIONS[name])
    for step in range(3):
        ids = batch(learner, 24, 100, seed=20 + step)
        learner.step(*(x.cuda() for x in ids[:3]), 0.003, offsets=None if ids[3] is None else ids[3].cuda())
    corpus = learner.corpus()
    assert float((corpus.float().norm(dim=-1) - 1).abs().max()) < 2.0 ** -8
    if name == "all":
        ids = batch(learner, 12, 50, seed=3)
        prob = learner.problem(ids[0].cuda(), offsets=ids[3].cuda(), corpus=corpus)
    else:
        prob = learner.problem(torch.arange(12, dtype=torch.int32, device="cuda"))
    assert torch.equal(prob.tensors[1], corpus)
    s, i = mol.topk_exact(prob, k)
    names = ("Q", "X", "a_q", "a_x", "W1", "b1", "W2", "b2")
    arrays = {n: (t.cpu().view(torch.int16).numpy().view("u2") if t.dtype == torch.bfloat16 else t.cpu().numpy())
              for n, t in zip(names, prob.tensors)}
    phi = mo.mol_scores(mo.Problem.from_arrays(dict(arrays, dtype="bf16")), list(range(12)))
    for b in range(12):
        check_topk_row(phi[b], i[b].cpu().numpy(), s[b].cpu().numpy(), k, f"trained query {b}")


def test_refusals():
    learner, plain = make(20, 90, 4, 4, 24, 32, seed=1, **OPTIONS["all"]), make(20, 90, 4, 4, 24, 32, seed=1)
    ids = [x.cuda() for x in batch(learner, 6, 40, seed=1)]
    before = [t.clone() for t in everything(learner)]
    for call in (lambda: learner.step(*ids[:3], 0.01), lambda: plain.step(*ids[:3], 0.01, offsets=ids[3]),
                 lambda: learner.step(*ids[:3], 0.01, offsets=ids[3].long()), lambda: learner.step(*ids[:3], 0.01, offsets=ids[3][:1]),
                 lambda: learner.problem(ids[0]), lambda: plain.states(ids[0], ids[3]), lambda: plain.advance(torch.zeros(1), ids[0]),
                 lambda: make(20, 90, 4, 4, 24, 32, seed=1, dropout=1.0), lambda: make(20, 90, 4, 4, 24, 32, seed=1, dropout=-0.1)):
        with pytest.raises(ValueError):
            call()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, everything(learner)))
    g = torch.zeros(20, 4, 24, device="cuda")
    with pytest.raises(ValueError):
        mol.Learner(*(plain.master[n] for n in NAMES), gates=g[:, :3].contiguous())
    with pytest.raises(ValueError):
        mol.Learner(*(plain.master[n] for n in NAMES), norm=(g.view(-1)[:96], g.view(-1)[:95]))


def test_a_history_without_events_moves_no_weights():
    """Its state is zero, so that with beta = 0 its components have no length: neither it nor they reach gamma and beta."""
    grads = []
    for lens, events in (([3, 0, 5], None), ([3, 2, 5], -1)):
        learner = make(20, 90, 4, 4, 24, 32, seed=1, **OPTIONS["all"])
        learner.master["beta"].zero_()
        learner.dropout = 0.0
        ids = torch.arange(1, 11, dtype=torch.int32) % 7
        offsets = torch.tensor([0, 3, 3 + lens[1], 8 + lens[1]], dtype=torch.int32)
        ids = torch.cat([ids[:3], torch.full((lens[1],), -1, dtype=torch.int32), ids[3:8]])
        _, items, target, _ = batch(learner, 8, 40, seed=4)
        loss = learner.step(ids.cuda(), items.cuda(), target[:3].cuda(), 0.01, offsets=offsets.cuda())
        assert torch.isfinite(loss).all()
        for n in ("gamma", "beta", "queries", "gates"):
            assert torch.isfinite(learner.grad[n]).all() and float(learner.grad[n].abs().max()) < 1e3, n
        grads.append({n: learner.grad[n].clone() for n in learner.grad})
    assert all(torch.equal(grads[0][n], grads[1][n]) for n in ("gamma", "beta", "queries", "gates", "items"))
