"""The learning operators where buffers end, where they are not aligned and
where offsets pass 32 bits (MI355X only)."""
import pytest
import torch

import learn_helpers as lh
from paper_2407_15462_amd import mol
from parity_helpers import log

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
NAMES = ("dQ", "dX", "da_q", "da_x", "dW1", "db1", "dW2", "db2")
GUARD = 512                                              # bytes on either side, 0xA5


class Guarded:
    """Tensors in buffers of their own with a band of known bytes before and behind."""

    def __init__(self):
        self.all = []

    def __call__(self, shape, dtype, fill=0xFF, offset=0):
        size = torch.empty((), dtype=dtype).element_size()
        n = size
        for s in shape:
            n *= s
        buf = torch.full((2 * GUARD + n + offset,), 0xA5, dtype=torch.uint8, device="cuda")
        body = buf[GUARD + offset:GUARD + offset + n]
        body.fill_(fill)
        self.all.append((buf, GUARD + offset, n))
        return body.view(dtype).view(shape)

    def check(self):
        for buf, at, n in self.all:
            assert bool((buf[:at] == 0xA5).all()) and bool((buf[at + n:] == 0xA5).all()), "written outside"


def off_by_one(t):
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    flat[1:] = t.reshape(-1)
    return flat[1:].view(t.shape)


# ------------------------------------------------------------------ buffers' ends
SHAPES = [(1, 1, 1, 1, 1, 1), (3, 21, 2, 3, 9, 7), (7, 50, 5, 3, 33, 24), (9, 70, 8, 8, 31, 64), (5, 37, 8, 8, 64, 64),
          (2, 19, 3, 7, 40, 100), (33, 129, 4, 4, 24, 32), (9, 40, 4, 4, 768, 64), (8, 33, 8, 8, 200, 64), (10, 20, 8, 4, 777, 33),
          (9, 41, 8, 4, 128, 128), (17, 50, 3, 2, 20, 70), (4, 33, 4, 4, 64, 96), (1, 40, 5, 4, 33, 127)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,N,Pq,Px,d,H", SHAPES)
def test_score_grad_keeps_to_its_buffers(B, N, Pq, Px, d, H, dtype):
    """A workspace of the stated size that holds NaN, outputs between guards, at addresses that only their type
    aligns: the bits of the plain call."""
    log(f"[edges] score_grad B={B} N={N} P={Pq}x{Px} d={d} H={H} {dtype}")
    inputs, dphi = lh.mol_inputs(B, N, Pq, Px, d, H, dtype, seed=3, device="cuda")
    prob = mol.Problem(*inputs)
    want = mol.score_grad(prob, dphi)
    g = Guarded()
    ws = g((mol.mol_workspace_size(prob, mol.MOL_OP_SCORE_GRAD),), torch.uint8)
    out = {n: g(tuple(t.shape), t.dtype, offset=t.element_size()) for n, t in zip(NAMES, inputs)}
    mol.score_grad(prob, dphi, ws=ws, out=out)
    g.check()
    for n in NAMES:
        assert torch.equal(out[n], want[n]), n
    for n in NAMES:                                      # each alone, in a workspace that the last call left behind
        one = {n: g(tuple(want[n].shape), want[n].dtype)}
        assert torch.equal(mol.score_grad(prob, dphi, ws=ws, only=(n,), out=one)[n], want[n]), n
    g.check()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,N,Pq,Px,d,H", SHAPES)
def test_score_grad_of_unaligned_tensors(B, N, Pq, Px, d, H, dtype):
    """Every tensor of the problem, and dphi, one element past an aligned address."""
    inputs, dphi = lh.mol_inputs(B, N, Pq, Px, d, H, dtype, seed=4)
    want, bound = lh.score_grads(inputs, dphi)
    got = mol.score_grad(mol.Problem(*(off_by_one(t.cuda()) for t in inputs)), off_by_one(dphi.cuda()))
    for n in NAMES:
        lh.within(got[n], want[n], bound[n], n)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_score_grad_does_not_mix_rows(dtype):
    """A NaN in an item's row reaches no other item's rows of the gradient, one in a query's row no other query's."""
    inputs, dphi = lh.mol_inputs(6, 45, 4, 4, 24, 32, dtype, seed=9, device="cuda")
    want = mol.score_grad(mol.Problem(*inputs), dphi)
    last = [t.clone() for t in inputs]
    last[1][:, 44] = float("nan")                        # the last item: what rows past the end repeat
    got = mol.score_grad(mol.Problem(*last), dphi)
    assert torch.equal(got["dX"][:, :44], want["dX"][:, :44]) and torch.equal(got["da_x"][:44], want["da_x"][:44])
    last = [t.clone() for t in inputs]
    last[0][5] = float("nan")                            # the last query
    got = mol.score_grad(mol.Problem(*last), dphi)
    assert torch.equal(got["dQ"][:5], want["dQ"][:5]) and torch.equal(got["da_q"][:5], want["da_q"][:5])


@pytest.mark.parametrize("C,V,d,T", [(1, 1, 1, 1), (3, 40, 33, 500), (2, 777, 64, 4097), (1, 5000, 8, 20000)])
@pytest.mark.parametrize("to", [F32, BF16])
def test_embedding_calls_keep_to_their_buffers(C, V, d, T, to):
    gen = torch.Generator().manual_seed(T)
    ids = torch.randint(-1, V + 1, (T,), generator=gen).int().cuda()
    grad = torch.randn(C, T, d, generator=gen).cuda()
    table = torch.randn(C, V, d, generator=gen).cuda()
    g = Guarded()
    size = torch.empty((), dtype=to).element_size()
    for offset in (0, size):
        out = mol.embed_lookup(table, ids, 0.5, out=g((C, T, d), to, offset=offset))
        assert torch.equal(out, mol.embed_lookup(table, ids, 0.5, dtype=to))
        ws = g((max(mol.mol_embed_grad_workspace(C, V, d, T), 1),), torch.uint8)
        got = mol.embed_grad(grad, ids, V, 0.5, ws=ws, out=g((C, V, d), to, offset=offset))
        # (rows at unaligned addresses are summed by other lanes in the same order of tokens or another)
        want, bound = lh.embed_grad(grad, ids, V, 0.5)
        lh.within(got, want, bound + lh.HALF[to] * want.abs() * 1.001 + lh.U * want.abs(), "sums")
    g.check()


@pytest.mark.parametrize("B,N", [(1, 1), (5, 63), (3, 2177), (2, 8705), (2, 34817), (1, 200001)])
def test_softmax_loss_keeps_to_its_buffers(B, N):
    gen = torch.Generator().manual_seed(N)
    phi = torch.randn(B, N, generator=gen).cuda()
    ids = torch.randint(-1, 5 * N, (N,), generator=gen).int().cuda()
    target = torch.randint(0, N, (B,), generator=gen).int().cuda()
    want = mol.softmax_loss(phi, target, ids, 5.0)
    g = Guarded()
    n = mol.mol_softmax_loss_workspace(B, N)
    ws = g((n,), torch.uint8) if n else None
    dphi, loss = g((B, N), F32, offset=4), g((B,), F32, offset=4)
    mol.mol_softmax_loss(phi, target, ids, 5.0, None, loss, dphi, ws)
    assert torch.equal(loss, want[0]) and torch.equal(dphi, want[1])
    # over the scores themselves
    own = g((B, N), F32, offset=4)
    own.copy_(phi)
    mol.softmax_loss(own, target, ids, 5.0, dphi=own, ws=ws)
    assert torch.equal(own, want[1])
    g.check()


@pytest.mark.parametrize("n", [1, 255, 257, 4096, 4097])
@pytest.mark.parametrize("eight", [False, True])
def test_adamw_keeps_to_its_buffers(n, eight):
    gen = torch.Generator().manual_seed(n)
    g = Guarded()

    def held(t, offset):
        out = g(tuple(t.shape), t.dtype, offset=offset)
        out.view(torch.uint8).copy_(t.cuda().view(torch.uint8))
        return out

    blocks = (n + 255) // 256
    p, gr = torch.randn(n, generator=gen), torch.randn(n, generator=gen).bfloat16()
    state = [torch.zeros(n, dtype=E4M3 if eight else F32) for _ in range(2)]
    scale = [torch.zeros(blocks) for _ in range(2)]
    got = []
    for offset in (0, 1):
        k = lambda t: held(t, offset * t.element_size())  # noqa: E731
        a = [[k(p)], [k(gr)], [k(state[0])], [k(state[1])]]
        s = [[k(scale[0])], [k(scale[1])]] if eight else [None, None]
        copy = g((n,), BF16, offset=2 * offset)
        mol.adamw_step(mol.AdamwTensors(*a, *s, weight_decay=0.1, out=dict(copy=[copy])), lr=0.01, seed=5)
        assert torch.equal(copy, a[0][0].bfloat16())
        got.append([a[0][0], a[2][0].view(torch.uint8), a[3][0].view(torch.uint8)])
    assert all(torch.equal(x, y) for x, y in zip(*got))
    g.check()


# ------------------------------------------------------------------ offsets past 32 bits
@pytest.mark.parametrize("N", [(1 << 24) - 12, (1 << 24) + 500])
def test_score_grad_of_a_corpus_past_32_bits(N):
    """a_x and da_x of 2^30 elements, 2^32 bytes: an item's gradients are those it has among few."""
    B, Pq, Px, d, H, some = 2, 8, 8, 8, 16, 1000
    log(f"[edges] score_grad N={N} P={Pq}x{Px}")
    gen = torch.Generator(device="cuda").manual_seed(1)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    Q, W1, W2 = randn(B, Pq, d).bfloat16(), (0.3 * randn(H, 64)).bfloat16(), (0.3 * randn(64, H)).bfloat16()
    X = torch.empty(Px, N, d, dtype=BF16, device="cuda").normal_(0, 0.3, generator=gen)
    a_q, b1, b2 = randn(B, 64), randn(H), randn(64)
    a_x = torch.empty(N, 64, device="cuda").normal_(0, 0.3, generator=gen)
    dphi = torch.empty(B, N, device="cuda").normal_(0, 1, generator=gen)
    got = mol.score_grad(mol.Problem(Q, X, a_q, a_x, W1, b1, W2, b2), dphi, only=("dX", "da_x", "dQ"))
    for n0 in (0, N // 2 + 3, N - some):
        part = [t.contiguous() for t in (X[:, n0:n0 + some], a_x[n0:n0 + some], dphi[:, n0:n0 + some])]
        inputs = [t.cpu() for t in (Q, part[0], a_q, part[1], W1, b1, W2, b2)]
        want, bound = lh.score_grads(inputs, part[2].cpu())
        lh.within(got["dX"][:, n0:n0 + some], want["dX"], bound["dX"], f"dX from {n0}")
        lh.within(got["da_x"][n0:n0 + some], want["da_x"], bound["da_x"], f"da_x from {n0}")
    assert bool(torch.isfinite(got["dQ"]).all())


@pytest.mark.parametrize("dtype,H", [(F32, 20), (BF16, 20), (BF16, 100)])
def test_score_grad_of_the_most_queries(dtype, H):
    """65,535 queries, slabs of the fewest items: a query's gradients are those it has among few, a sum's parts add up."""
    B, N, Pq, Px, d = 65535, 70, 8, 4, 24
    log(f"[edges] score_grad B={B} N={N} H={H} {dtype}")
    gen = torch.Generator(device="cuda").manual_seed(4)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    P = Pq * Px
    Q, X = (0.3 * randn(B, Pq, d)).to(dtype), (0.3 * randn(Px, N, d)).to(dtype)
    a_q, a_x, b1, b2 = randn(B, P), randn(N, P), randn(H), randn(P)
    W1, W2 = (0.3 * randn(H, P)).to(dtype), (0.3 * randn(P, H)).to(dtype)
    dphi = randn(B, N)
    dphi[4:-4] = 0                                       # (so that the sums over queries are those of eight)
    got = mol.score_grad(mol.Problem(Q, X, a_q, a_x, W1, b1, W2, b2), dphi)
    rows = [0, 1, 2, 3, B - 4, B - 3, B - 2, B - 1]
    want, bound = lh.score_grads([t.cpu() for t in (Q[rows], X, a_q[rows], a_x, W1, b1, W2, b2)], dphi[rows].cpu())
    for n in NAMES:
        lh.within(got[n][rows] if n in ("dQ", "da_q") else got[n], want[n], bound[n], n)
    assert int((got["dQ"][4:-4] != 0).sum()) == 0 and int((got["da_q"][4:-4] != 0).sum()) == 0


def test_softmax_loss_past_32_bits():
    """Score rows that begin past 2^32 elements."""
    B, N = 61000, 70417
    log(f"[edges] softmax_loss B={B} N={N}")
    phi = torch.zeros(B, N, device="cuda")
    rows = [0, (1 << 32) // N, B - 1]
    gen = torch.Generator().manual_seed(2)
    few = torch.randn(3, N, generator=gen)
    phi[rows] = few.cuda()
    target = torch.full((B,), 5, dtype=torch.int32, device="cuda")
    loss, dphi = mol.softmax_loss(phi, target, inv_temp=2.0, dphi=phi)
    z = 2.0 * few.double()
    want = torch.logsumexp(z, 1) - z[:, 5]
    pi = torch.softmax(z, 1)
    pi[:, 5] -= 1
    # sums of 70,417 weights in chains of at most 300 and a tree above, e^z to a few 2^-24, the loss to 20
    assert float((loss[rows].double().cpu() - want).abs().max()) < 420 * lh.U
    assert float(((dphi[rows].double().cpu() - 2 * pi).abs() / (2 * pi).abs()).max()) < 400 * lh.U * 2
    # a row of equal scores
    assert float((loss[B // 2].double() - torch.log(torch.tensor(float(N), dtype=torch.float64))).abs()) < 420 * lh.U


def test_adamw_past_32_bits():
    """The last blocks of 2^32 + 300 elements: the bits of a small call that starts at their place."""
    n, tail = (1 << 32) + 300, 812                       # the last 812: from a multiple of 256
    log(f"[edges] adamw n={n}")
    gen = torch.Generator().manual_seed(3)
    blocks = (n + 255) // 256
    p = torch.zeros(n, dtype=BF16, device="cuda")
    g = torch.zeros(n, dtype=BF16, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    ms, vs = (torch.zeros(blocks, device="cuda") for _ in range(2))
    p[-tail:], g[-tail:] = torch.randn(tail, generator=gen).bfloat16().cuda(), torch.randn(tail, generator=gen).bfloat16().cuda()
    small = [t[-tail:].clone() for t in (p, g, m.view(torch.uint8), v.view(torch.uint8))]
    small[2:] = [t.view(E4M3) for t in small[2:]]
    sms, svs = (torch.zeros(4, device="cuda") for _ in range(2))
    assert (n - tail) % 256 == 0
    mol.adamw_step(mol.AdamwTensors([p], [g], [m], [v], [ms], [vs], weight_decay=0.1), lr=0.1, seed=9)
    plan = mol.AdamwTensors(*([t] for t in small), [sms], [svs], weight_decay=0.1)
    plan.c[0].rng_offset = n - tail
    mol.adamw_step(plan, lr=0.1, seed=9)
    for a, b in zip((p, m.view(torch.uint8), v.view(torch.uint8)), (small[0], small[2].view(torch.uint8), small[3].view(torch.uint8))):
        assert torch.equal(a[-tail:], b)
    assert torch.equal(ms[-4:], sms) and torch.equal(vs[-4:], svs)
    assert int((p[:4096] != 0).sum()) == 0


# ------------------------------------------------------------------ graphs
def test_two_graphs_share_a_workspace():
    """Two captured sequences that use one workspace, replayed in turn with eager work and new inputs between them:
    the bits of eager calls."""
    B, N, Pq, Px, d, H, V = 24, 9000, 4, 4, 32, 32, 500
    inputs, dphi = lh.mol_inputs(B, N, Pq, Px, d, H, BF16, seed=2, device="cuda")
    prob = mol.Problem(*inputs)
    gen = torch.Generator().manual_seed(7)
    ids = torch.randint(-1, V, (N,), generator=gen).int().cuda()
    phi = torch.randn(3, 50000, generator=gen).cuda()
    target = torch.tensor([1, 40000, 7], dtype=torch.int32, device="cuda")
    sizes = (mol.mol_workspace_size(prob, mol.MOL_OP_SCORE_GRAD), mol.mol_embed_grad_workspace(Px, V, d, N),
             mol.mol_softmax_loss_workspace(3, 50000))
    ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")

    def first():
        g = mol.score_grad(prob, dphi, ws=ws)
        return list(g.values()) + [mol.embed_grad(g["dX"], ids, V, ws=ws)]

    def second():
        return list(mol.softmax_loss(phi, target, inv_temp=3.0, ws=ws)) + [mol.embed_grad(prob.tensors[1], ids, V, 2.0, ws=ws)]

    graphs = []
    for run in (first, second):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        graphs.append((graph, out, run))
    for turn in range(3):
        dphi.mul_(1.5)
        phi.add_(0.25)
        ids.copy_(ids.roll(11))
        for graph, out, run in graphs:
            for t in out:
                t.zero_()
            ws.fill_(0xFF)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            held = [t.clone() for t in out]
            for got, want in zip(held, run()):
                assert torch.equal(got, want), turn
