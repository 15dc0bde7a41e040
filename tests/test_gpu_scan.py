"""The gated recurrence over histories, its gradient and its single step, against
plain float64 forms (MI355X only).  Bounds follow from counts of float32 roundings
(rows_helpers)."""
import itertools

import pytest
import torch

import rows_helpers as rh
from learn_helpers import within
from paper_2407_15462_amd import mol
from parity_helpers import log
from test_gpu_rows import fenced, off_by_one, unharmed

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
NAME = {F32: "f32", BF16: "bf16"}
TYPES = [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)]

# lengths of histories; rows in front of the first and behind the last
SETS = {
    "one": ([1], 0, 0), "pair": ([2], 0, 0), "none": ([0], 0, 3), "edges": ([128, 0, 0, 128, 64, 64, 1, 127, 0], 0, 0),
    "mixed": ([0, 3, 0, 17, 1, 1, 200, 0, 64, 129, 15, 16, 33, 0], 5, 9), "long": ([5000], 0, 0), "behind": ([30], 700, 900),
    "many": ([1, 0, 2, 5, 0, 0, 3] * 150, 2, 1),
}


# (the long sets, whose oracle takes its time, for some sizes and types only)
CASES = [(name, d, ti, to) for name in SETS for d in (1, 2, 8, 9, 33, 64, 65, 128, 300) for ti, to in TYPES
         if name not in ("long", "many") or (d not in (1, 8, 33, 128) and ti == to)]


def make(lens, front, back, d, dtype, seed=0):
    T = front + sum(lens) + back
    g = torch.Generator().manual_seed(T * 7 + d + seed)
    gate = (2 + 2 * torch.randn(T, d, generator=g)).to(dtype)
    x = torch.randn(T, d, generator=g).to(dtype)
    dead = torch.ones(T, dtype=torch.bool)
    dead[front:T - back if back else T] = False
    gate[dead] = float("nan")                                    # rows of no history may hold anything
    x[dead] = float("inf")
    offsets = torch.tensor(list(itertools.accumulate([front] + lens)), dtype=torch.int32)
    h0 = torch.randn(len(lens), d, generator=g)
    return gate.cuda(), x.cuda(), offsets.cuda(), h0.cuda(), dead


@pytest.mark.parametrize("name,d,ti,to", CASES)
def test_scan(name, d, ti, to):
    lens, front, back = SETS[name]
    log(f"[scan] {name} d={d} {NAME[ti]}->{NAME[to]}")
    gate, x, offsets, h0, dead = make(lens, front, back, d, ti)
    T, B = x.shape[0], len(lens)
    for start in (h0, None):
        want, bound, live, last, lb = rh.gated_scan(gate, x, lens, front, start, to)
        out, buf = fenced((T, d), to)
        end, ebuf = fenced((B, d), F32)
        mol.gated_scan(gate, x, offsets, h0=start, out=out, last=end)
        within(out[live.cuda()], want[live], bound[live], "h")
        within(end, last, lb, "last")
        assert unharmed(buf, T * d) and unharmed(ebuf, B * d)
        assert bool((out[dead.cuda()] == 77).all()), "rows of no history were written"
        h, e = mol.gated_scan(off_by_one(gate), off_by_one(x), offsets, h0=start, dtype=to)
        assert torch.equal(h[live.cuda()], out[live.cuda()]) and torch.equal(e, end), "unaligned rows or a second run differ"
    s = h0.clone()
    h, e = mol.gated_scan(gate, x, offsets, h0=s, dtype=to, last=s)
    want, end = mol.gated_scan(gate, x, offsets, h0=h0, dtype=to)
    assert e is s and torch.equal(s, end) and torch.equal(h[live.cuda()], want[live.cuda()]), "states in place differ"


@pytest.mark.parametrize("name,d,ti,th", CASES)
def test_scan_grad(name, d, ti, th):
    lens, front, back = SETS[name]
    log(f"[scan_grad] {name} d={d} x {NAME[ti]} h {NAME[th]}")
    gate, x, offsets, h0, dead = make(lens, front, back, d, ti)
    T, B = x.shape[0], len(lens)
    g = torch.Generator().manual_seed(d)
    dh = torch.randn(T, d, generator=g).to(th).cuda()
    dh[dead.cuda()] = float("nan")
    dlast = torch.randn(B, d, generator=g).cuda()
    live = ~dead
    on = live.cuda()
    for start, a, b in ((h0, dh, dlast), (None, dh, None), (h0, None, dlast)):
        h = torch.full((T, d), float("nan"), dtype=th, device="cuda")
        mol.gated_scan(gate, x, offsets, h0=start, out=h)
        want = rh.gated_scan_grad(gate, x, h, a, lens, front, start, b, ti)
        got = mol.gated_scan_grad(gate, x, h, dh=a, offsets=offsets, h0=start, dlast=b)
        within(got[0][on], want[0][0][live], want[0][1][live], "dgate")
        within(got[1][on], want[1][0][live], want[1][1][live], "dx")
        assert not got[0][~on].any() and not got[1][~on].any(), "rows of no history have gradients"
        if start is None:
            assert got[2] is None
        else:
            within(got[2], *want[2], "dh0")
        again = mol.gated_scan_grad(off_by_one(gate), off_by_one(x), off_by_one(h), dh=None if a is None else off_by_one(a),
                                    offsets=offsets, h0=start, dlast=b)
        assert all(p is None or torch.equal(p, q) for p, q in zip(got, again)), "unaligned rows or a second run differ"


@pytest.mark.parametrize("d,T", [(130, 40000), (8, 150000), (64, 40001), (7, 70001)])
@pytest.mark.parametrize("t", [F32, BF16])
def test_one_long_history(d, T, t):
    """Chunks and groups of chunks that wait for each other, against the scan in pieces and itself."""
    log(f"[scan] one history T={T} d={d} {NAME[t]}")
    g = torch.Generator().manual_seed(T)
    gate = (6 + torch.randn(T, d, generator=g)).to(t).cuda()            # states kept over hundreds of tokens
    x, h0 = torch.randn(T, d, generator=g).to(t).cuda(), torch.randn(1, d, generator=g).cuda()
    dh = torch.randn(T, d, generator=g).to(t).cuda()
    want, bound, _, last, lb = rh.gated_scan(gate, x, [T], 0, h0, F32)
    h, end = mol.gated_scan(gate, x, h0=h0, dtype=F32)
    within(h, want, bound, "h")
    within(end, last, lb, "last")
    got = mol.gated_scan_grad(gate, x, h.to(t), dh=dh, h0=h0)
    ref = rh.gated_scan_grad(gate, x, h.to(t), dh, [T], 0, h0, None, t)
    for name, a, b in zip(("dgate", "dx", "dh0"), got, ref):
        within(a, *b, name)
    for _ in range(5):
        h2, end2 = mol.gated_scan(gate, x, h0=h0, dtype=F32)
        assert torch.equal(h2, h) and torch.equal(end2, end), "two runs differ"
        assert all(torch.equal(a, b) for a, b in zip(got, mol.gated_scan_grad(gate, x, h.to(t), dh=dh, h0=h0))), "two runs differ"


@pytest.mark.parametrize("d", [3, 64, 200])
def test_a_historys_nan_stays_in_it(d):
    lens = [40, 300, 500, 1, 90]
    gate, x, offsets, h0, _ = make(lens, 0, 0, d, F32)
    clean, end = mol.gated_scan(gate, x, offsets, h0=h0)
    dh = torch.ones_like(x)
    cg = mol.gated_scan_grad(gate, x, clean, dh=dh, offsets=offsets, h0=h0)
    a, b = 340, 840                                               # the third history
    for what in ("nan", "inf"):
        y, e = x.clone(), dh.clone()
        y[a + 200] = float(what)
        e[a + 200] = float(what)
        h, last = mol.gated_scan(gate, y, offsets, h0=h0)
        assert not torch.isfinite(h[a + 200]).any()
        keep = torch.ones(len(x), dtype=torch.bool, device="cuda")
        keep[a + 200:b] = False
        assert torch.equal(h[keep], clean[keep]) and torch.equal(last[[0, 1, 3, 4]], end[[0, 1, 3, 4]])
        got = mol.gated_scan_grad(gate, x, clean, dh=e, offsets=offsets, h0=h0)
        keep[:] = True
        keep[a:a + 201] = False
        assert all(torch.equal(p[keep], q[keep]) for p, q in zip(got[:2], cg[:2]))
        assert not torch.isfinite(got[1][a + 200]).any() and torch.equal(got[2][[0, 1, 3, 4]], cg[2][[0, 1, 3, 4]])


def test_gates_far_out():
    gate = torch.tensor([[-200.0, -90.0, -30.0, 30.0, 90.0, 200.0, float("inf"), float("-inf")]] * 3, device="cuda")
    x = torch.full_like(gate, 3.0)
    h0 = torch.full((1, 8), 2.0, device="cuda")
    h, last = mol.gated_scan(gate, x, h0=h0)
    want = torch.tensor([3.0, 3, 3, 2, 2, 2, 2, 3]).expand(3, 8)
    within(h, want, 1e-6, "h")
    dg, dx, dh0 = mol.gated_scan_grad(gate, x, h, dh=torch.ones_like(x), h0=h0)
    assert torch.isfinite(dg).all() and torch.isfinite(dx).all()
    within(dh0[0], torch.tensor([0.0, 0, 0, 3, 3, 3, 3, 0]), 1e-6, "dh0")


def test_offsets_are_clamped():
    """Offsets past either end count as that end."""
    gate, x, offsets, h0, _ = make([100, 57], 0, 0, 70, F32)
    want = mol.gated_scan(gate, x, offsets, h0=h0)
    out = offsets.clone()
    out[0], out[2] = -9, 1 << 30
    got = mol.gated_scan(gate, x, out, h0=h0)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    a = mol.gated_scan_grad(gate, x, want[0], dh=x, offsets=offsets, h0=h0)
    b = mol.gated_scan_grad(gate, x, want[0], dh=x, offsets=out, h0=h0)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_no_tokens():
    x = torch.empty(0, 20, device="cuda")
    off, h0 = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.randn(3, 20, device="cuda")
    h, last = mol.gated_scan(x, x, off, h0=h0)
    assert h.shape == (0, 20) and torch.equal(last, h0)
    assert not mol.gated_scan(x, x, off)[1].any()
    assert torch.equal(mol.gated_scan_grad(x, x, x, offsets=off, h0=h0, dlast=h0 + 1)[2], h0 + 1)


@pytest.mark.parametrize("T", [60, 3000])
def test_mostly_empty_histories(T):
    """Far more histories than tokens: each one's state, in one chunk and in several."""
    B, d = 5001, 140
    g = torch.Generator().manual_seed(T)
    offsets = torch.sort((torch.rand(B + 1, generator=g) * (T + 1)).int().clamp(max=T)).values
    offsets[0], offsets[-1] = 0, T
    lens = (offsets[1:] - offsets[:-1]).tolist()
    gate, x = (torch.randn(T, d, generator=g).cuda() for _ in range(2))
    h0 = torch.randn(B, d, generator=g)
    want, bound, _, last, lb = rh.gated_scan(gate, x, lens, 0, h0, F32)
    h, end = mol.gated_scan(gate, x, offsets.cuda(), h0=h0.cuda())
    within(h, want, bound, "h")
    within(end, last, lb, "last")
    dlast = torch.randn(B, d, generator=g)
    ref = rh.gated_scan_grad(gate, x, h, None, lens, 0, h0, dlast, F32)
    for name, a, b in zip(("dgate", "dx", "dh0"), mol.gated_scan_grad(gate, x, h, offsets=offsets.cuda(), h0=h0.cuda(), dlast=dlast.cuda()), ref):
        within(a, *b, name)


def test_gradient_is_the_difference_quotient():
    lens, d, h = [3, 0, 9], 5, 1e-3
    g = torch.Generator().manual_seed(2)
    T = sum(lens)
    gate, x, dh = (torch.randn(T, d, generator=g) for _ in range(3))
    h0, dlast = torch.randn(3, d, generator=g), torch.randn(3, d, generator=g)
    off = torch.tensor([0, 3, 3, 12], dtype=torch.int32).cuda()

    def loss(gate, x, h0):
        hs, _, _, last, _ = rh.gated_scan(gate, x, lens, 0, h0, F32)
        return float((hs * dh.double()).sum() + (last * dlast.double()).sum())

    state, _ = mol.gated_scan(gate.cuda(), x.cuda(), off, h0=h0.cuda())
    got = mol.gated_scan_grad(gate.cuda(), x.cuda(), state, dh=dh.cuda(), offsets=off, h0=h0.cuda(), dlast=dlast.cuda())
    args = [gate.double(), x.double(), h0.double()]
    for k, grad in enumerate(got):
        for i in range(args[k].numel()):
            step = torch.zeros(args[k].numel(), dtype=torch.float64)
            step[i] = h
            up, down = list(args), list(args)
            up[k], down[k] = args[k] + step.view_as(args[k]), args[k] - step.view_as(args[k])
            # (the quotient is off by h^2 / 6 times a third derivative, which stays below 10 here)
            assert abs(float(grad.flatten()[i]) - (loss(*up) - loss(*down)) / (2 * h)) < 1e-5, (k, i)


@pytest.mark.parametrize("B,d", [(1, 1), (3, 5), (256, 512), (33, 77), (4096, 64)])
@pytest.mark.parametrize("ti,to", TYPES)
def test_step(B, d, ti, to):
    log(f"[step] B={B} d={d} {NAME[ti]}->{NAME[to]}")
    gate, x, _, h0, _ = make([1] * B, 0, 0, d, ti)
    want, bound, _, last, lb = rh.gated_scan(gate, x, [1] * B, 0, h0, to)
    new, buf = fenced((B, d), F32)
    out, obuf = fenced((B, d), to)
    keep = h0.clone()
    assert mol.gated_step(gate, x, h0, new=new, out=out) is out
    within(out, want, bound, "h")
    within(new, last, lb, "state")
    assert torch.equal(h0, keep) and unharmed(buf, B * d) and unharmed(obuf, B * d)
    got = mol.gated_step(off_by_one(gate), off_by_one(x), h0, dtype=to)
    assert torch.equal(got, out) and torch.equal(h0, new), "in place or unaligned differs"


def test_prefill_then_steps_are_the_scan():
    """A history in one scan, and as a prefill and single steps: the same states up to their roundings."""
    d, T = 96, 90
    gate, x, _, h0, _ = make([T], 0, 0, d, F32)
    want, bound, _, last, lb = rh.gated_scan(gate, x, [T], 0, h0[:1], F32)
    _, state = mol.gated_scan(gate[:60].contiguous(), x[:60].contiguous(), h0=h0[:1].contiguous())
    for t in range(60, T):
        h = mol.gated_step(gate[t:t + 1].contiguous(), x[t:t + 1].contiguous(), state)
        within(h[0], want[t], bound[t], f"h of token {t}")
    within(state, last, lb, "last")


def test_graphs_that_share_a_workspace():
    lens = [700, 0, 3, 2500, 64, 1]
    gate, x, offsets, h0, _ = make(lens, 0, 0, 150, BF16)
    gate2, x2, offsets2, h02, _ = make([900, 800], 4, 5, 100, BF16)
    ws = mol.gated_scan_workspace(x, len(lens))
    dh = torch.randn(x.shape, device="cuda").bfloat16()

    def one(ws):
        h, last = mol.gated_scan(gate, x, offsets, h0=h0, ws=ws)
        return (h, last) + mol.gated_scan_grad(gate, x, h, dh=dh, offsets=offsets, h0=h0, dlast=last, ws=ws)

    def two(ws):
        h = torch.zeros_like(x2)
        return mol.gated_scan(gate2, x2, offsets2, h0=h02, out=h, ws=ws)

    one(ws), two(ws)
    graphs, held = [], []
    for f in (one, two):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            held.append(f(ws))
    for i in range(4):
        x.copy_(torch.randn(x.shape, device="cuda"))
        x2.copy_(torch.randn(x2.shape, device="cuda"))
        for k in (0, 1, 0) if i % 2 else (1, 0):
            graphs[k].replay()
        torch.cuda.synchronize()
        for k, f in enumerate((one, two)):
            assert all(torch.equal(a, b) for a, b in zip(held[k], f(None))), f"replay {i} of graph {k}"


def test_two_streams_at_once():
    gate, x, offsets, h0, _ = make([3000, 1, 2000], 0, 0, 256, F32)
    want = mol.gated_scan(gate, x, offsets, h0=h0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [[mol.gated_scan(gate, x, offsets, h0=h0, stream=s) for _ in range(4)] for s in streams]
    torch.cuda.synchronize()
    for g in got:
        for h, last in g:
            assert torch.equal(h, want[0]) and torch.equal(last, want[1])


def test_indices_past_32_bits():
    """More than 2^31 elements: the last histories are as scanned alone."""
    d, n, B = 520, 1000, 4200
    T = n * B
    assert T * d > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(5)
    gate, x = torch.empty(T, d, dtype=BF16, device="cuda"), torch.empty(T, d, dtype=BF16, device="cuda")
    gate.normal_(2, 1, generator=g)
    x.normal_(0, 1, generator=g)
    offsets = torch.arange(B + 1, dtype=torch.int32, device="cuda") * n
    h, last = mol.gated_scan(gate, x, offsets)
    dg, dx, _ = mol.gated_scan_grad(gate, x, h, dh=x, offsets=offsets)
    for b in (0, B // 2, B - 1):
        rows = slice(b * n, b * n + n)
        gb, xb, hb = gate[rows].contiguous(), x[rows].contiguous(), h[rows].contiguous()
        want, bound, _, end, lb = rh.gated_scan(gb, xb, [n], 0, None, BF16)
        within(hb, want, bound, f"h of history {b}")
        within(last[b:b + 1], end, lb, f"last of history {b}")
        ref = rh.gated_scan_grad(gb, xb, hb, xb, [n], 0, None, None, BF16)
        within(dg[rows], *ref[0], f"dgate of history {b}")
        within(dx[rows], *ref[1], f"dx of history {b}")


def test_workspaces_serve_smaller_scans():
    gate, x, offsets, h0, _ = make([300, 5000, 0, 70], 0, 0, 200, BF16)
    ws = mol.gated_scan_workspace(torch.empty(9000, 300, device="cuda"), 9)
    ws.fill_(0xFF)                                       # what an earlier call left: words that say they are there
    want = mol.gated_scan(gate, x, offsets, h0=h0)
    got = mol.gated_scan(gate, x, offsets, h0=h0, ws=ws)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    small = mol.gated_scan(gate[:900, :64].contiguous(), x[:900, :64].contiguous(), ws=ws)
    assert all(torch.equal(a, b) for a, b in zip(small, mol.gated_scan(gate[:900, :64].contiguous(), x[:900, :64].contiguous())))
