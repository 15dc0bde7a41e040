"""Embedding rows and their gradient, the sampled-softmax loss, the gradient
of the scores and AdamW against plain float64 forms (MI355X only).  Bounds
follow from counts of float32 roundings (learn_helpers)."""
import numpy as np
import pytest
import torch

import learn_helpers as lh
from oracle import mol_oracle as mo
from paper_2407_15462_amd import mol
from parity_helpers import log

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
NAME = {F32: "f32", BF16: "bf16"}


def rand_ids(T, V, gen, empties=True):
    """Popular ids many times, some empty slots."""
    ids = (V * torch.rand(T, generator=gen).double() ** 3).long().clamp_(max=V - 1)
    if empties and T > 3:
        ids[torch.rand(T, generator=gen) < 0.1] = -1
        ids[T // 2] = V                                  # past the table
    return ids.int()


def off_by_one(t):
    """The same values from an address that is only element-aligned."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    flat[1:] = t.reshape(-1)
    return flat[1:].view(t.shape)


# ------------------------------------------------------------------ lookup
@pytest.mark.parametrize("C,V,d,T", [(1, 1, 1, 1), (1, 7, 3, 5), (2, 50, 33, 64), (4, 1000, 64, 300), (8, 333, 32, 1),
                                     (1, 100, 1024, 17), (3, 41, 129, 1000), (1, 5, 65536, 3), (2, 4000, 8, 70000)])
@pytest.mark.parametrize("ti,to", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_lookup(C, V, d, T, ti, to):
    log(f"[lookup] C={C} V={V} d={d} T={T} {NAME[ti]}->{NAME[to]}")
    gen = torch.Generator().manual_seed(C * 1000 + d + T)
    table = torch.randn(C, V, d, generator=gen).to(ti).cuda()
    ids = rand_ids(T, V, gen).cuda()
    table[:, 0, 0] = float("nan")                        # (an empty slot does not read row 0)
    ok = (ids >= 0) & (ids < V)
    for scale in (1.0, 2.75):
        # one float32 product, one rounding: the same bits as torch's
        want = torch.where(ok[None, :, None], table[:, ids.long().clamp(0, V - 1)].float() * scale, 0.0).to(to)
        for tab in (table, off_by_one(table)):
            got = mol.embed_lookup(tab, ids, scale, dtype=to)
            assert torch.equal(torch.nan_to_num(got, nan=7.0), torch.nan_to_num(want, nan=7.0))
    out = off_by_one(torch.empty(C, T, d, dtype=to, device="cuda"))
    mol.embed_lookup(table, ids, 2.75, out=out)
    assert torch.equal(torch.nan_to_num(out, nan=7.0), torch.nan_to_num(want, nan=7.0))


def test_lookup_of_no_ids():
    out = mol.embed_lookup(torch.ones(2, 3, 4, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"))
    assert out.shape == (2, 0, 4)


# ------------------------------------------------------------------ gradient of the lookup
@pytest.mark.parametrize("C,V,d,T", [(1, 1, 1, 1), (1, 3, 5, 40), (2, 50, 33, 64), (4, 1000, 64, 300), (1, 9, 1024, 130),
                                     (2, 300, 96, 4096), (1, 5000, 32, 4097), (8, 2000, 32, 9000), (1, 70000, 8, 30000),
                                     (2, 3000, 16, 16384), (1, 999, 8, 16385), (1, 500, 4, 65537), (1, 9, 4, 15), (1, 9, 4, 17),
                                     (2, 5, 8, 65), (1, 1, 4, 1000), (1, 300, 16, 8192), (2, 77, 8, 8193),
                                     (1, 1 << 21, 4, 6000), (1, 40, 64, 50000), (1, 3, 1000, 777), (1, 2, 65536, 9)])
@pytest.mark.parametrize("ti,to", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_embed_grad(C, V, d, T, ti, to):
    log(f"[embed_grad] C={C} V={V} d={d} T={T} {NAME[ti]}->{NAME[to]}")
    gen = torch.Generator().manual_seed(C * 1000 + d + T)
    grad = torch.randn(C, T, d, generator=gen).to(ti).cuda()
    ids = rand_ids(T, V, gen).cuda()
    want, bound = lh.embed_grad(grad, ids, V, 1.25)
    bound = bound + lh.HALF[to] * want.abs() * 1.001
    got = mol.embed_grad(grad, ids, V, 1.25, dtype=to)
    lh.within(got, want, bound, "sums")
    assert torch.equal(got, mol.embed_grad(grad, ids, V, 1.25, dtype=to)), "two runs differ"
    got1 = mol.embed_grad(off_by_one(grad), ids, V, 1.25, dtype=to)
    lh.within(got1, want, bound, "sums of unaligned rows")
    # added to what is there; rows without tokens keep their bits
    base = torch.randn(C, V, d, generator=gen).to(to).cuda()
    out = base.clone()
    mol.embed_grad(grad, ids, V, 1.25, out=out, accumulate=True)
    seen = torch.zeros(V, dtype=torch.bool)
    seen[ids.cpu().long()[(ids.cpu() >= 0) & (ids.cpu() < V)]] = True
    assert torch.equal(out[:, ~seen], base[:, ~seen])
    total = want + base.double().cpu()
    lh.within(out[:, seen], total[:, seen], (bound + lh.HALF[to] * total.abs() * 1.001 + lh.U * total.abs())[:, seen], "added")


@pytest.mark.parametrize("T", [1, 200, 6000])
def test_embed_grad_of_one_row_and_of_none(T):
    grad = torch.randn(2, T, 24, generator=torch.Generator().manual_seed(T)).cuda()
    ids = torch.full((T,), 4, dtype=torch.int32, device="cuda")
    want, bound = lh.embed_grad(grad, ids, 6, 1.0)
    lh.within(mol.embed_grad(grad, ids, 6), want, bound + lh.U * want.abs(), "one row")
    assert bool((mol.embed_grad(grad, ids.fill_(-1), 6) == 0).all())
    out = torch.full((2, 6, 24), 3.0, device="cuda")
    mol.embed_grad(grad[:, :0].contiguous(), ids[:0], 6, out=out, accumulate=True)
    assert bool((out == 3.0).all())
    mol.embed_grad(grad[:, :0].contiguous(), ids[:0], 6, out=out)
    assert bool((out == 0.0).all())


def test_embed_grad_is_the_transpose_of_lookup():
    """<lookup(E), G> = <E, grad(G)>, by differences in E: the lookup is linear."""
    gen = torch.Generator().manual_seed(3)
    E, G = torch.randn(3, 90, 40, generator=gen).cuda(), torch.randn(3, 500, 40, generator=gen).cuda()
    ids = rand_ids(500, 90, gen).cuda()
    D = torch.randn(3, 90, 40, generator=gen).cuda()
    up = (mol.embed_lookup(E + D, ids, 0.5).double() * G.double()).sum()
    down = (mol.embed_lookup(E - D, ids, 0.5).double() * G.double()).sum()
    dot = (mol.embed_grad(G, ids, 90, 0.5).double() * D.double()).sum()
    size = (mol.embed_lookup(E.abs() + D.abs(), ids, 0.5).double() * G.double().abs()).sum()
    # E +- D rounded once, the products once; grad's rows of at most 500 sums
    assert abs((up - down) / 2 - dot) <= size * 505 * lh.U


def test_rows_past_32_bits():
    """Tables whose rows lie beyond 2^32 bytes and 2^32 elements from their start."""
    V, d = (1 << 30) + 7, 4
    table = torch.zeros(1, V, d, dtype=BF16, device="cuda")
    far = torch.tensor([V - 1, 0, 1 << 29, V - 3, V, -1, V - 1], dtype=torch.int32, device="cuda")
    rows = torch.arange(1, 29, device="cuda").view(7, 4).to(BF16)
    live = [0, 1, 2, 3]
    table[0, far[live].long()] = rows[live]
    got = mol.embed_lookup(table, far, 2.0)
    want = rows * 2
    want[[4, 5]] = 0
    want[6] = want[0]
    assert torch.equal(got[0], want)
    table.fill_(9.0)
    mol.embed_grad(rows.view(1, 7, 4), far, V, out=table)
    sums = rows.float()
    sums[0] += sums[6]
    assert torch.equal(table[0, far[live].long()], sums[live].to(BF16))
    assert int((table != 0).sum()) == 16


# ------------------------------------------------------------------ loss
def loss_case(B, N, gen, with_ids):
    phi = torch.randn(B, N, generator=gen).clamp_(-3, 3)
    target = torch.randint(0, N, (B,), generator=gen).int()
    if B > 2:
        target[1], target[2] = -1, N
    ids = None
    if with_ids:
        ids = torch.randint(0, max(2, N // 2), (N,), generator=gen).int()
        ids[torch.rand(N, generator=gen) < 0.1] = -5
    return phi, target, ids


@pytest.mark.parametrize("B,N", [(1, 1), (3, 2), (5, 63), (4, 64), (7, 1000), (2, 2048), (3, 2049), (4, 8193), (3, 32768),
                                 (2, 36865), (1, 100003), (130, 129), (600, 40000)])
@pytest.mark.parametrize("with_ids", [False, True])
def test_softmax_loss(B, N, with_ids):
    log(f"[loss] B={B} N={N} ids={with_ids}")
    gen = torch.Generator().manual_seed(B * 7 + N)
    phi, target, ids = loss_case(B, N, gen, with_ids)
    weight = torch.rand(B, generator=gen)
    dev = [None if t is None else t.cuda() for t in (phi, target, ids, weight)]
    for inv_temp, w in ((1.0, None), (20.0, weight)):
        want = lh.softmax_loss(phi, target, ids, inv_temp, w)
        loss, dphi = mol.softmax_loss(dev[0], dev[1], dev[2], inv_temp, None if w is None else dev[3])
        lh.within(loss, want[0], want[2], "loss")
        lh.within(dphi, want[1], want[3], "dphi")
    buf = dev[0].clone()
    again, same = mol.softmax_loss(buf, dev[1], dev[2], 20.0, dev[3], dphi=buf)
    assert same is buf and torch.equal(buf, dphi) and torch.equal(again, loss)


@pytest.mark.parametrize("N", [70, 9000, 50000])
def test_softmax_loss_of_what_masked_columns_hold(N):
    """NaN, infinities and the lowest value in left-out columns change no bit; kept ones follow the formula."""
    gen = torch.Generator().manual_seed(N)
    phi, target, _ = loss_case(6, N, gen, False)
    target = torch.tensor([0, 3, 5, 7, 9, 11]).int()
    ids = torch.arange(N).int()
    out = torch.tensor([20, 33, 41, N - 2])
    ids[out] = -1
    ids[50] = ids[3]                                      # a copy of row 1's positive
    clean = [t.clone() for t in mol.softmax_loss(phi.cuda(), target.cuda(), ids.cuda(), 2.0)]
    dirty = phi.clone()
    dirty[:, out] = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(F32).min])
    dirty[1, 50] = float("nan")
    loss, dphi = mol.softmax_loss(dirty.cuda(), target.cuda(), ids.cuda(), 2.0)
    assert torch.equal(loss, clean[0]) and torch.equal(dphi, clean[1])
    assert float(dphi[1, 50]) == 0.0
    # a kept -inf (and the lowest value) takes no part, a kept NaN poisons its row alone
    phi[0, 60], phi[2, 61], phi[3, 62] = -float("inf"), float("nan"), torch.finfo(F32).min
    loss, dphi = mol.softmax_loss(phi.cuda(), target.cuda(), ids.cuda(), 2.0)
    assert bool(torch.isnan(loss[2])) and float(dphi[0, 60]) == 0.0 and float(dphi[3, 62]) == 0.0
    good = torch.tensor([0, 1, 3, 4, 5])
    want = lh.softmax_loss(phi[good], target[good], ids, 2.0, None)
    lh.within(loss[good.cuda()], want[0], want[2], "loss")
    lh.within(dphi[good.cuda()], want[1], want[3], "dphi")
    # nothing but the positive is left: loss 0, gradient 0 but for rounding
    ids.fill_(-1)
    ids[target[4].item()] = 8
    loss, dphi = mol.softmax_loss(phi.cuda(), target.cuda(), ids.cuda(), 2.0)
    assert loss.tolist()[4] == 0.0 and bool((dphi == 0).all()) and bool((loss == 0).all())


def test_softmax_loss_against_differences():
    gen = torch.Generator().manual_seed(9)
    phi, target, ids = loss_case(8, 300, gen, True)
    _, dphi = mol.softmax_loss(phi.cuda(), target.cuda(), ids.cuda(), 3.0)
    h = 1e-5
    for _ in range(3):
        D = torch.randn(8, 300, generator=gen).double()
        f = [lh.softmax_loss(phi.double() + k * h * D, target, ids, 3.0, None)[0].sum() for k in (1, -1)]
        # differences: h^2 |D|^3 inv_temp^3 of truncation, 1e-16 / h of rounding
        assert abs((f[0] - f[1]) / (2 * h) - (dphi.double().cpu() * D).sum()) < 1e-4


# ------------------------------------------------------------------ gradient of the scores
GRAD_SHAPES = [(1, 1, 1, 1, 1, 1), (3, 5, 1, 1, 16, 4), (2, 17, 2, 3, 24, 20), (5, 33, 4, 4, 64, 32), (4, 64, 8, 2, 32, 16),
               (9, 70, 8, 4, 64, 64), (6, 131, 8, 8, 32, 64), (13, 40, 8, 8, 64, 64), (2, 20, 4, 4, 768, 64), (7, 50, 3, 5, 40, 130),
               (3, 35, 64, 1, 16, 24), (3, 35, 1, 64, 33, 256), (5, 20, 7, 9, 17, 100), (4, 40, 8, 4, 128, 128)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,N,Pq,Px,d,H", GRAD_SHAPES)
def test_score_grad(B, N, Pq, Px, d, H, dtype):
    log(f"[score_grad] B={B} N={N} P={Pq}x{Px} d={d} H={H} {NAME[dtype]}")
    inputs, dphi = lh.mol_inputs(B, N, Pq, Px, d, H, dtype, seed=B + N + d)
    want, bound = lh.score_grads(inputs, dphi)
    prob = mol.Problem(*(t.cuda() for t in inputs))
    got = mol.score_grad(prob, dphi.cuda())
    for name in want:
        lh.within(got[name], want[name], bound[name], name)
    again = mol.score_grad(prob, dphi.cuda())
    assert all(torch.equal(got[n], again[n]) for n in got), "two runs differ"
    some = mol.score_grad(prob, dphi.cuda(), only=("dW1", "da_x"))
    assert set(some) == {"dW1", "da_x"} and torch.equal(some["dW1"], got["dW1"]) and torch.equal(some["da_x"], got["da_x"])


@pytest.mark.parametrize("B,N,Pq,Px,d,H,dtype", [(300, 500, 8, 8, 64, 64, BF16), (70, 900, 4, 4, 64, 32, F32),
                                                 (130, 260, 8, 4, 128, 128, BF16)])
def test_score_grad_over_many_tiles(B, N, Pq, Px, d, H, dtype):
    log(f"[score_grad] B={B} N={N} P={Pq}x{Px} d={d} H={H} {NAME[dtype]}")
    inputs, dphi = lh.mol_inputs(B, N, Pq, Px, d, H, dtype, seed=77)
    want, bound = lh.score_grads(inputs, dphi)
    got = mol.score_grad(mol.Problem(*(t.cuda() for t in inputs)), dphi.cuda())
    for name in want:
        lh.within(got[name], want[name], bound[name], name)


def test_score_grad_in_slabs():
    """A corpus whose pairs pass the workspace's buffer is taken in slabs: the sums over slabs are those of the parts."""
    B, N, Pq, Px, d, H = 1024, 2500, 8, 8, 16, 16
    inputs, dphi = lh.mol_inputs(B, N, Pq, Px, d, H, BF16, seed=5, device="cuda")
    got = mol.score_grad(mol.Problem(*inputs), dphi)
    Q, X, a_q, a_x, W1, b1, W2, b2 = inputs
    # float64 by parts of 50 items on the GPU, with the derivative taken by torch
    want = [torch.zeros_like(t, dtype=torch.float64) for t in inputs]
    for n0 in range(0, N, 50):
        part = [t.double() for t in (Q, X[:, n0:n0 + 50], a_q, a_x[n0:n0 + 50], W1, b1, W2, b2)]
        part = [t.clone().requires_grad_() for t in part]
        q, x, aq, ax, w1, c1, w2, c2 = part
        s = torch.matmul(q.reshape(1, B * Pq, d), x.transpose(1, 2)).view(Px, B, Pq, 50).permute(1, 3, 2, 0).reshape(-1, Pq * Px)
        hid = torch.nn.functional.silu(s @ w1.t() + c1)
        lg = (hid @ w2.t() + c2).view(B, 50, -1) + aq[:, None] + ax[None]
        phi = (torch.softmax(lg, -1) * s.view(B, 50, -1)).sum(-1)
        for k, gr in enumerate(torch.autograd.grad(phi, part, dphi[:, n0:n0 + 50].double())):
            if k == 1:
                want[k][:, n0:n0 + 50] = gr
            elif k == 3:
                want[k][n0:n0 + 50] = gr
            else:
                want[k] += gr
    for name, w in zip(("dQ", "dX", "da_q", "da_x", "dW1", "db1", "dW2", "db2"), want):
        rel = float((got[name].double() - w).norm() / w.norm())
        # one bf16 rounding is off by 2^-8 / sqrt(3) at most in the root mean square; float32 chains of this length by under 1e-5
        assert rel < (2.0 ** -8 if got[name].dtype == BF16 else 1e-5), (name, rel)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_score_grad_of_few_queries_and_many_items(dtype):
    """Sums of dQ and the weights over 200,003 items with B P_q of 6: many splits of a short product."""
    B, N, Pq, Px, d, H, part = 3, 200003, 2, 1, 1024, 16, 20000
    log(f"[score_grad] B={B} N={N} P={Pq}x{Px} d={d} H={H} {NAME[dtype]}")
    inputs, dphi = lh.mol_inputs(B, N, Pq, Px, d, H, dtype, seed=8, device="cuda")
    got = mol.score_grad(mol.Problem(*inputs), dphi)
    Q, X, a_q, a_x, W1, b1, W2, b2 = inputs
    want = [torch.zeros_like(t, dtype=torch.float64) for t in inputs]
    for n0 in range(0, N, part):
        leaves = [t.double().clone().requires_grad_() for t in (Q, X[:, n0:n0 + part], a_q, a_x[n0:n0 + part], W1, b1, W2, b2)]
        q, x, aq, ax, w1, c1, w2, c2 = leaves
        s = torch.matmul(q.reshape(B * Pq, d), x[0].t()).view(B, Pq, -1).transpose(1, 2)
        lg = torch.nn.functional.silu(s @ w1.t() + c1) @ w2.t() + c2 + aq[:, None] + ax[None]
        phi = (torch.softmax(lg, -1) * s).sum(-1)
        for k, gr in enumerate(torch.autograd.grad(phi, leaves, dphi[:, n0:n0 + part].double())):
            (want[k][:, n0:n0 + part] if k == 1 else want[k][n0:n0 + part] if k == 3 else want[k]).add_(gr)
    for name, w in zip(("dQ", "dX", "da_q", "da_x", "dW1", "db1", "dW2", "db2"), want):
        rel = float((got[name].double() - w).norm() / w.norm())
        # a bf16 rounding: 2^-8 / sqrt(3) at most; in float32 a pair's terms take about ten roundings (6e-7) and the
        # sums, of 2000 terms in a chain at most, sqrt(2000) 2^-24 = 2.7e-6 more
        assert rel < (2.0 ** -8 if got[name].dtype == BF16 else 1e-5), (name, rel)


def test_score_grad_against_differences_of_the_oracle():
    inputs, dphi = lh.mol_inputs(4, 30, 4, 2, 24, 16, F32, seed=21)
    got = mol.score_grad(mol.Problem(*(t.cuda() for t in inputs)), dphi.cuda())
    names = ("Q", "X", "a_q", "a_x", "W1", "b1", "W2", "b2")
    gen = torch.Generator().manual_seed(4)

    def value(arrays):
        p = mo.Problem.from_arrays(dict({n: np.asarray(a) for n, a in zip(names, arrays)}, dtype="f32"))
        return float((np.asarray(mo.mol_scores(p, list(range(4)))) * dphi.double().numpy()).sum())

    base = [t.numpy() for t in inputs]
    h = 1e-3
    for k, name in enumerate(names):
        D = torch.randn(inputs[k].shape, generator=gen).double().numpy()
        D *= h / np.linalg.norm(D)
        # float32 points, which the oracle takes as they are; their distance is what counts
        up, down = (base[k] + D).astype(np.float32), (base[k] - D).astype(np.float32)
        f = [value([x if i == k else a for i, a in enumerate(base)]) for x in (up, down)]
        dot = float((got["d" + name].double().cpu().numpy() * (up.astype(np.float64) - down)).sum())
        # third derivatives are of order one here: h^3 of truncation; float32's 1e-5 of the gradient
        assert abs((f[0] - f[1]) - dot) < 2 * h ** 3 + 1e-5 * abs(dot), name


# ------------------------------------------------------------------ AdamW
def adamw_tensors(sizes, pt, gt, eight, gen):
    p = [(0.1 * torch.randn(n, generator=gen)).to(pt).cuda() for n in sizes]
    g = [(1e-3 * torch.randn(n, generator=gen)).to(gt).cuda() for n in sizes]
    if not eight:
        return p, g, [(1e-4 * torch.randn(n, generator=gen)).cuda() for n in sizes], \
            [(1e-3 * torch.randn(n, generator=gen).cuda()) ** 2 for n in sizes], None, None
    blocks = [(n + 255) // 256 for n in sizes]
    codes = lambda n, lo, hi: torch.randint(lo, hi, (n,), generator=gen).to(torch.uint8)  # noqa: E731
    m = [((torch.randint(0, 2, (n,), generator=gen) << 7).to(torch.uint8) | codes(n, 0, 0x7F)).view(E4M3).cuda() for n in sizes]
    v = [codes(n, 1, 0x7F).view(E4M3).cuda() for n in sizes]
    ms = [(1e-6 * torch.rand(b, generator=gen)).cuda() for b in blocks]
    vs = [(1e-6 * torch.rand(b, generator=gen)).cuda() for b in blocks]
    return p, g, m, v, ms, vs


def wide(q, scale):
    """Values of 8-bit states."""
    return q.float().double().cpu() * scale.double().cpu().repeat_interleave(256)[:q.numel()]


def check_one(before, after, pt, eight, lr, b1, b2, eps, decay, step, scale, copy, i):
    p, g, m, v, ms, vs = before
    p2, m2, v2, ms2, vs2 = after
    n = p.numel()
    m0 = wide(m, ms) if eight else m.double().cpu()
    v0 = wide(v, vs) ** 2 if eight else v.double().cpu()
    wp, wm, wv = lh.adamw(p, g, m0, v0, lr, b1, b2, eps, decay, step, scale)
    gg = g.double().cpu().abs() * abs(scale)
    pd = p.double().cpu()
    # decoding a state is one rounding (v: of its square, three); m' and v' have
    # three more of each term; the update takes those, relative to its terms, and
    # at most sixteen others (root, reciprocal, products, rates)
    em = 6 * lh.U * (b1 * m0.abs() + (1 - b1) * gg) + 1e-44
    ev = 10 * lh.U * wv + 1e-44
    per = lr / (1 - b1 ** step) / ((wv / (1 - b2 ** step)).sqrt() + eps)
    ep = per * em + 24 * lh.U * per * wm.abs() + 4 * lh.U * pd.abs()
    lh.within(p2, wp, ep + lh.HALF[pt] * wp.abs() * 1.001, f"p[{i}]")
    if copy is not None:
        lh.within(copy, wp, ep + lh.HALF[BF16] * wp.abs() * 1.001, f"copy[{i}]")
    if not eight:
        lh.within(m2, wm, em, f"m[{i}]")
        lh.within(v2, wv, ev, f"v[{i}]")
        return
    for q, s, w in ((m2, ms2, wm), (v2, vs2, wv.sqrt())):
        pad = torch.zeros((n + 255) // 256 * 256, dtype=torch.float64)
        pad[:n] = w
        top = pad.view(-1, 256).abs().amax(1)
        lh.within(s, top / 448, top * 12 * lh.U, f"scale[{i}]")
        y = w / top.clamp(min=1e-300).repeat_interleave(256)[:n] * 448
        spacing = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        # one of the two neighbours of the value (a value that a few float32
        # roundings move over a code counts from there), or up from zero
        lh.within(q.float(), y, spacing * 1.001 + 1e-4, f"codes[{i}]")
    assert not bool(((v2.float().cpu() == 0) & (wv > 0)).any()), "a positive v is stored as zero"


SIZES = [1, 255, 256, 257, 0, 5000, 4096, 4097, 3, 70001]


@pytest.mark.parametrize("eight", [False, True], ids=["f32states", "e4m3states"])
@pytest.mark.parametrize("pt,gt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_adamw(pt, gt, eight):
    log(f"[adamw] p {NAME[pt]} g {NAME[gt]} 8-bit states: {eight}")
    gen = torch.Generator().manual_seed(11)
    before = adamw_tensors(SIZES, pt, gt, eight, gen)
    p, g, m, v, ms, vs = before
    decay = [0.1 * (i % 2) for i in range(len(SIZES))]
    scale = torch.tensor([0.5], device="cuda")
    new = lambda ts: None if ts is None else [torch.zeros_like(t) for t in ts]  # noqa: E731
    out = dict(p=new(p), m=new(m), v=new(v), m_scale=new(ms), v_scale=new(vs),
               copy=[None if i % 3 == 1 else torch.zeros_like(t, dtype=BF16) for i, t in enumerate(p)])
    keep = [t.clone() for ts in (p, m, v) for t in ts]
    plan = mol.AdamwTensors(p, g, m, v, ms, vs, weight_decay=decay, out=out)
    args = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, step=3, seed=5, grad_scale=scale)
    mol.adamw_step(plan, **args)
    assert all(torch.equal(a.view(torch.uint8) if a.dtype == E4M3 else a, b.view(torch.uint8) if b.dtype == E4M3 else b)
               for a, b in zip(keep, [t for ts in (p, m, v) for t in ts])), "the old state was written"
    after = (out["p"], out["m"], out["v"], out["m_scale"], out["v_scale"])
    for i in range(len(SIZES)):
        check_one([t and t[i] for t in before], [t and t[i] for t in after], pt, eight, 1e-2, 0.9, 0.999, 1e-8, decay[i], 3, 0.5,
                  out["copy"][i], i)
    # in place: the same bits; lr and step read on the GPU: the same bits
    for dev in (False, True):
        q = [[t.clone() for t in ts] if ts is not None else None for ts in (p, m, v, ms, vs)]
        plan = mol.AdamwTensors(q[0], g, q[1], q[2], q[3], q[4], weight_decay=decay)
        if dev:
            args.update(lr=torch.tensor([1e-2], device="cuda"), step=torch.tensor([3], dtype=torch.int32, device="cuda"))
        mol.adamw_step(plan, **args)
        for a, b in zip(q[0] + q[1] + q[2], after[0] + after[1] + after[2]):
            if a.dtype == E4M3:
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
            elif dev:                                     # (lr as float32 before the division: one rounding more)
                lh.within(a, b, 2 * lh.HALF[a.dtype] * b.abs().double().cpu() + 1e-9, "rates from the GPU")
            else:
                assert torch.equal(a, b)


def test_adamw_rounding_is_right_on_average():
    """The mean of the stored states over many elements of one value is that value: 2^16 random bits of 2^16 elements leave
    a standard error of half a code / 256."""
    n = 1 << 16
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 3.3e-4, device="cuda")
    g[::256] = 1.0e-3                                      # the blocks' largest
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4M3), torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4M3)
    ms, vs = torch.zeros(n // 256, device="cuda"), torch.zeros(n // 256, device="cuda")
    for seed, step in ((0, 1), (1, 1), (0, 2)):
        out = dict(p=[p.clone()], m=[torch.zeros_like(m)], v=[torch.zeros_like(v)], m_scale=[ms.clone()], v_scale=[vs.clone()])
        mol.adamw_step(mol.AdamwTensors([p], [g], [m], [v], [ms], [vs], out=out), step=step, seed=seed)
        small = torch.ones(n, dtype=torch.bool)
        small[::256] = False
        for q, s, want in ((out["m"][0], out["m_scale"][0], 0.1 * 3.3e-4), (out["v"][0], out["v_scale"][0], (1e-3 ** 0.5) * 3.3e-4)):
            got = wide(q, s)[small]
            code = float(got.max() - got.min())
            assert 0 < code < 0.13 * want and abs(float(got.mean()) - want) < 5 * code / 2 / 256


def test_adamw_first_step_and_lost_blocks():
    """States of zeros; a gradient of zeros leaves p but for its decay; a NaN poisons its own block alone."""
    n = 1000
    p = torch.randn(n, generator=torch.Generator().manual_seed(1)).cuda()
    g = torch.zeros(n, device="cuda")
    codes = lambda: torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4M3)  # noqa: E731
    m, v, ms, vs = codes(), codes(), torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda")
    q = p.clone()
    mol.adamw_step(mol.AdamwTensors([q], [g], [m], [v], [ms], [vs], weight_decay=0.5), lr=0.5)
    assert torch.equal(q, p * 0.75) and bool((ms == 0).all()) and bool((m.float() == 0).all())
    g[300] = float("nan")
    mol.adamw_step(mol.AdamwTensors([q], [g], [m], [v], [ms], [vs]), lr=0.5, step=2)
    assert bool(torch.isnan(q[300])) and int(torch.isnan(q).sum()) == 1
    assert torch.isnan(ms).tolist() == [False, True, False, False] == torch.isnan(vs).tolist()


def test_adamw_over_many_tensors_is_each_alone():
    gen = torch.Generator().manual_seed(2)
    sizes = [int(x) for x in torch.randint(1, 3000, (77,), generator=gen)]
    p, g, m, v, _, _ = adamw_tensors(sizes, F32, BF16, False, gen)
    alone = [[t.clone() for t in ts] for ts in (p, m, v)]
    mol.adamw_step(mol.AdamwTensors(p, g, m, v, weight_decay=0.01), step=7)
    for i in range(len(sizes)):
        mol.adamw_step(mol.AdamwTensors([alone[0][i]], [g[i]], [alone[1][i]], [alone[2][i]], weight_decay=0.01), step=7)
    for a, b in zip(alone, (p, m, v)):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_adamw_of_unaligned_tensors():
    gen = torch.Generator().manual_seed(6)
    for eight in (False, True):
        p, g, m, v, ms, vs = adamw_tensors([3001], F32, BF16, eight, gen)
        q = [[off_by_one(t) if t.dtype != E4M3 else off_by_one(t.view(torch.uint8)).view(E4M3) for t in ts] for ts in (p, g, m, v)]
        s = [None if t is None else [t[0].clone()] for t in (ms, vs)]
        mol.adamw_step(mol.AdamwTensors(p, g, m, v, ms, vs), step=2)
        mol.adamw_step(mol.AdamwTensors(*q, *s), step=2)
        assert torch.equal(p[0], q[0][0])
        assert torch.equal(m[0].view(torch.uint8), q[2][0].view(torch.uint8))


# ------------------------------------------------------------------ streams
def test_another_stream_than_the_current():
    """Inputs made on one stream, the calls on another: results equal those on the current stream."""
    inputs, dphi = lh.mol_inputs(20, 300, 4, 4, 64, 32, BF16, seed=8, device="cuda")
    ids = torch.randint(0, 50, (300,)).int().cuda()
    grad = torch.randn(4, 300, 64, device="cuda")
    phi = torch.randn(20, 300, device="cuda")
    target = torch.arange(20).int().cuda()
    prob = mol.Problem(*inputs)

    def run(stream):
        return (mol.embed_lookup(grad, ids, 2.0, stream=stream), mol.embed_grad(grad, ids, 50, stream=stream),
                *mol.softmax_loss(phi, target, ids, stream=stream), *mol.score_grad(prob, dphi, stream=stream).values())

    want = run(None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(side)
    got2 = run(side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, got2))
