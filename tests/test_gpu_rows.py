"""Layer norm, L2 normalisation and dropout, forwards and back, against plain
float64 forms (MI355X only).  Bounds follow from counts of float32 roundings
(rows_helpers)."""
import pytest
import torch

import rows_helpers as rh
from learn_helpers import within
from paper_2407_15462_amd import mol
from parity_helpers import log

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
NAME = {F32: "f32", BF16: "bf16"}
TYPES = [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)]


def off_by_one(t):
    """The same values from an address that is only element-aligned."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    flat[1:] = t.reshape(-1)
    return flat[1:].view(t.shape)


def fenced(shape, dtype, value=77.0):
    """(a tensor, its buffer): elements around it that must stay as they are."""
    n = 1
    for s in shape:
        n *= s
    buf = torch.full((n + 34,), value, dtype=dtype, device="cuda")
    return buf[17:17 + n].view(shape), buf


def unharmed(buf, n, value=77.0):
    return bool((buf[:17] == value).all()) and bool((buf[17 + n:] == value).all())


ROWS = [(1, 1), (5, 2), (3, 7), (70, 8), (33, 9), (64, 32), (100, 33), (17, 64), (9, 65), (130, 100), (7, 128), (40, 129),
        (5, 255), (3000, 48), (33, 512), (5, 777), (12, 1000), (3, 1024), (2, 1025), (6, 2048), (3, 4095), (2, 4096), (2, 4097),
        (3, 8192), (1, 16383), (2, 16384)]


def rows(T, d, dtype, seed=0):
    g = torch.Generator().manual_seed(1000 * T + d + seed)
    x = torch.randn(T, d, generator=g) * torch.exp(torch.randn(T, 1, generator=g)) + torch.randn(T, 1, generator=g)
    return x.to(dtype).cuda()


@pytest.mark.parametrize("T,d", ROWS)
@pytest.mark.parametrize("ti,to", TYPES)
def test_layer_norm(T, d, ti, to):
    log(f"[layer_norm] T={T} d={d} {NAME[ti]}->{NAME[to]}")
    x = rows(T, d, ti)
    g = torch.Generator().manual_seed(d)
    gamma, beta = (1 + 0.3 * torch.randn(d, generator=g)).cuda(), torch.randn(d, generator=g).cuda()
    for ga, be in ((gamma, beta), (None, None), (gamma, None)):
        want, bound = rh.layer_norm(x, ga, be, 1e-5, to)
        out, buf = fenced((T, d), to)
        assert mol.layer_norm(x, ga, be, out=out) is out
        within(out, want, bound, "y")
        assert unharmed(buf, T * d)
        got = mol.layer_norm(off_by_one(x), ga, be, dtype=to)
        assert torch.equal(got, out), "unaligned rows differ"
    if ti == to:
        y = x.clone()
        mol.layer_norm(y, gamma, None, out=y)
        assert torch.equal(y, out), "in place differs"


@pytest.mark.parametrize("T,d", ROWS)
@pytest.mark.parametrize("ti,tg", TYPES)
def test_layer_norm_grad(T, d, ti, tg):
    log(f"[layer_norm_grad] T={T} d={d} x {NAME[ti]} dy {NAME[tg]}")
    x, dy = rows(T, d, ti), rows(T, d, tg, seed=5)
    gamma = (1 + 0.3 * torch.randn(d, generator=torch.Generator().manual_seed(d))).cuda()
    for ga, to in ((gamma, F32), (None, BF16)):
        want, bound = rh.layer_norm_grad(dy, x, ga, 1e-5, to)
        out, buf = fenced((T, d), to)
        got = mol.layer_norm_grad(dy, x, ga, out=out)
        for name, a, b, c in zip(("dx", "dgamma", "dbeta"), got, want, bound):
            within(a, b, c, name)
        assert unharmed(buf, T * d)
        again = mol.layer_norm_grad(off_by_one(dy), off_by_one(x), ga, dtype=to)
        assert all(torch.equal(a, b) for a, b in zip(got, again)), "unaligned rows or a second run differ"
        alone = mol.layer_norm_grad(dy, x, ga, dtype=to, weights=False)
        assert torch.equal(alone[0], got[0]) and alone[1] is None and alone[2] is None
    if ti == BF16:
        y = x.clone()
        mol.layer_norm_grad(dy, y, None, out=y)
        assert torch.equal(y, got[0]), "in place differs"


def test_layer_norm_grad_over_many_rows():
    """Weights' gradients over more rows than a launch has workgroups: +-1 in dy, so that dbeta is exact."""
    T, d = 300001, 40
    g = torch.Generator().manual_seed(3)
    dy = (torch.randint(0, 2, (T, d), generator=g) * 2 - 1).float()
    x = torch.randn(T, d, generator=g)
    _, dgamma, dbeta = mol.layer_norm_grad(dy.cuda(), x.cuda())
    assert torch.equal(dbeta.cpu(), dy.sum(0))
    c = x.double() - x.double().mean(1, keepdim=True)
    xhat = c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt()
    # a lane adds 19 rows, then as above
    within(dgamma, (dy * xhat).sum(0), 160 * rh.U * xhat.abs().sum(0) + 60 * rh.U * T, "dgamma")


def test_norms_past_32_bits():
    """More than 2^31 elements: the last rows are as they are alone."""
    T, d = 4200001, 520
    x = torch.empty(T, d, dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    dy = x.flip(0)
    rows_ = [0, T // 2, T - 2, T - 1]
    some, dsome = x[rows_].contiguous(), dy[rows_].contiguous()
    assert torch.equal(mol.layer_norm(x)[rows_], mol.layer_norm(some))
    assert torch.equal(mol.normalize(x)[rows_], mol.normalize(some))
    assert torch.equal(mol.normalize_grad(dy, x)[rows_], mol.normalize_grad(dsome, some))
    dx, dgamma, dbeta = mol.layer_norm_grad(dy, x)
    assert torch.equal(dx[rows_], mol.layer_norm_grad(dsome, some)[0])
    # dbeta: a lane's 4102 rows at most, then as in the helpers, of magnitudes 0.8 on average
    assert float((dbeta.double() - dy.double().sum(0)).abs().max()) < (4102 + 128) * rh.U * T


def test_a_workspace_for_more_serves_fewer():
    ws = mol.layer_norm_grad_workspace(torch.empty(6000, 8192, device="cuda"))
    for T, d in ((6000, 4096), (5000, 4097), (6000, 30), (10, 8192)):
        x, dy = rows(T, d, BF16), rows(T, d, BF16, seed=1)
        ws.fill_(0x7F)
        assert all(torch.equal(a, b) for a, b in zip(mol.layer_norm_grad(dy, x, ws=ws), mol.layer_norm_grad(dy, x)))


def test_layer_norm_gradient_is_the_difference_quotient():
    T, d, h = 3, 21, 1e-3
    g = torch.Generator().manual_seed(8)
    x, dy, gamma = torch.randn(T, d, generator=g), torch.randn(T, d, generator=g), torch.randn(d, generator=g)
    dx, dgamma, dbeta = mol.layer_norm_grad(dy.cuda(), x.cuda(), gamma.cuda())

    def loss(x, gamma, beta):
        c = x - x.mean(1, keepdim=True)
        return (dy.double() * (c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt() * gamma + beta)).sum()

    beta = torch.zeros(d, dtype=torch.float64)
    for name, got, at in (("x", dx, 0), ("gamma", dgamma, 1), ("beta", dbeta, 2)):
        args = [x.double(), gamma.double(), beta]
        for i in range(args[at].numel()):
            step = torch.zeros(args[at].numel(), dtype=torch.float64)
            step[i] = h
            up, down = list(args), list(args)
            up[at], down[at] = args[at] + step.view_as(args[at]), args[at] - step.view_as(args[at])
            want = float(loss(*up) - loss(*down)) / (2 * h)
            # the quotient's own error is of h^2 times third derivatives, about 1e-6 times sums of |dy gamma| below 100
            assert abs(float(got.flatten()[i]) - want) < 2e-4, (name, i)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e15, 1e25, 1e37])
def test_norms_of_extreme_rows(scale):
    """Rows whose squares leave float32's range, beside ordinary ones."""
    for d in (9, 64, 300, 5000):
        x = rows(5, d, F32)
        x = x / x.abs().amax()
        x[1] *= scale
        x[3] *= scale
        dy = rows(5, d, F32, seed=2)
        want, bound = rh.layer_norm(x, None, None, 1e-5, F32)
        within(mol.layer_norm(x), want, bound + 1e-37, f"layer norm d={d}")
        want, bound = rh.normalize(x, 1e-35, F32)
        within(mol.normalize(x, eps=1e-35), want, bound, f"normalize d={d}")
        want, bound = rh.normalize_grad(dy, x, 1e-35, F32)
        within(mol.normalize_grad(dy, x, eps=1e-35), want, bound + 1e-44, f"normalize_grad d={d}")
        (want, _, _), (bound, _, _) = rh.layer_norm_grad(dy, x, None, 1e-5, F32)
        got = mol.layer_norm_grad(dy, x)[0]
        # (gradients of rows of 1e37 are below float32's normal numbers)
        within(got, want, bound + 1e-37, f"layer_norm_grad d={d}")


@pytest.mark.parametrize("T,d", ROWS)
@pytest.mark.parametrize("ti,to", TYPES)
def test_normalize(T, d, ti, to):
    log(f"[normalize] T={T} d={d} {NAME[ti]}->{NAME[to]}")
    x, dy = rows(T, d, ti), rows(T, d, to, seed=9)
    x[T // 2] = 0
    want, bound = rh.normalize(x, 1e-12, to)
    out, buf = fenced((T, d), to)
    mol.normalize(x, out=out)
    within(out, want, bound, "y")
    assert unharmed(buf, T * d)
    assert torch.equal(mol.normalize(off_by_one(x), dtype=to), out)
    x[T // 2] = 1e-3                                     # (rows of zeros have gradients of 1e12 dy)
    want, bound = rh.normalize_grad(dy, x, 1e-12, ti)
    out, buf = fenced((T, d), ti)
    mol.normalize_grad(dy, x, out=out)
    within(out, want, bound, "dx")
    assert unharmed(buf, T * d)
    assert torch.equal(mol.normalize_grad(off_by_one(dy), off_by_one(x)), out)


def test_normalize_below_eps():
    x = torch.tensor([[3e-3, 4e-3], [0.0, 0.0], [3.0, 4.0]], device="cuda")
    dy = torch.tensor([[1.0, 2.0], [5.0, -7.0], [1.0, 2.0]], device="cuda")
    within(mol.normalize(x, eps=0.01), torch.tensor([[0.3, 0.4], [0, 0], [0.6, 0.8]]), 1e-6, "y")
    # dy / eps where the row is within eps; (dy - y <y, dy>) / 5 = ([1, 2] - [0.6, 0.8] * 2.2) / 5 beyond
    within(mol.normalize_grad(dy, x, eps=0.01), torch.tensor([[100.0, 200], [500, -700], [-0.064, 0.048]]),
           torch.tensor([[1e-4], [1e-3], [1e-6]]), "dx")


def test_a_rows_nan_is_its_own():
    for d in (6, 64, 100, 2000):
        x, dy = rows(9, d, F32), rows(9, d, F32, seed=1)
        x[4, d // 2] = float("nan")
        dy[6, 0] = float("inf")
        for got, bad in ((mol.layer_norm(x), {4}), (mol.normalize(x), {4}), (mol.normalize_grad(dy, x), {4, 6}),
                         (mol.layer_norm_grad(dy, x)[0], {4, 6})):
            assert set(torch.nonzero(~torch.isfinite(got).all(1))[:, 0].tolist()) == bad


def test_norms_without_rows_and_shapes():
    x = torch.empty(0, 12, device="cuda")
    assert mol.layer_norm(x).shape == (0, 12) and mol.normalize(x).shape == (0, 12)
    dx, dgamma, dbeta = mol.layer_norm_grad(x, x)
    assert dx.shape == (0, 12) and not dgamma.any() and not dbeta.any()
    assert mol.normalize_grad(x, x).shape == (0, 12)
    y = rows(24, 16, F32)
    assert torch.equal(mol.normalize(y.view(2, 3, 4, 16)), mol.normalize(y).view(2, 3, 4, 16))
    assert torch.equal(mol.layer_norm(y[0]), mol.layer_norm(y)[0])


# ------------------------------------------------------------------ dropout
@pytest.mark.parametrize("n", [1, 7, 8, 9, 63, 64, 1000, 2048, 2049, 70001])
@pytest.mark.parametrize("ti,to", TYPES)
def test_dropout(n, ti, to):
    log(f"[dropout] n={n} {NAME[ti]}->{NAME[to]}")
    g = torch.Generator().manual_seed(n)
    x = (torch.randn(n, generator=g).abs() + 0.1).to(ti).cuda()
    res = torch.randn(n, generator=g).to(to).cuda()
    for p, seed, step, offset in ((0.2, 1, 0, 0), (0.5, 0x9E3779B97F4A7C15, 7, 1 << 40), (0.9, -3, 0xFFFFFFFF, (1 << 35) - 8),
                                  (0.0, 5, 1, 8), (65535 / 65536, 5, 1, 16)):
        keep, want, bound = rh.dropout(x, p, seed & (1 << 64) - 1, step, offset, None, to)
        out, buf = fenced((n,), to)
        mol.dropout(x, p, seed, step=step, offset=offset, out=out)
        assert torch.equal(out.cpu() != 0, keep)
        within(out, want, bound, "y")
        assert unharmed(buf, n)
        assert torch.equal(mol.dropout(off_by_one(x), p, seed, step=step, offset=offset, dtype=to), out)
        _, want, bound = rh.dropout(x, p, seed & (1 << 64) - 1, step, offset, res, to)
        # (of a sum that cancels, the bound counts the terms)
        got = mol.dropout(x, p, seed, step=step, offset=offset, residual=res)
        within(got, want, bound + 3 * rh.U * (x.double().cpu().abs() / (1 - p) + res.double().cpu().abs()), "y + residual")
        r = res.clone()
        assert torch.equal(mol.dropout(x, p, seed, step=step, offset=offset, residual=r, out=r), got)
        on = torch.tensor([step - (1 << 32) if step >= 1 << 31 else step], dtype=torch.int32, device="cuda")
        assert torch.equal(mol.dropout(x, p, seed, step=on, offset=offset, dtype=to), out)


def test_dropout_places_and_bits():
    """Pieces of a tensor at their places give the whole's mask; dropped NaN and infinities are zeros."""
    x = torch.ones(5000, device="cuda")
    whole = mol.dropout(x, 0.3, 11, step=4, offset=80)
    assert torch.equal(torch.cat([mol.dropout(x[a:b], 0.3, 11, step=4, offset=80 + a) for a, b in
                                  ((0, 8), (8, 1000), (1000, 1016), (1016, 5000))]), whole)
    bad = torch.where(whole == 0, float("nan"), 1.0)
    bad[torch.nonzero(whole == 0)[0]] = float("inf")
    assert torch.equal(mol.dropout(bad, 0.3, 11, step=4, offset=80), whole)
    # the generator's known answer for counter 0 and key 0: 6627e8d5 e169c58d bc57ac4c 9b00dbd8
    halves = [0xE8D5, 0x6627, 0xC58D, 0xE169, 0xAC4C, 0xBC57, 0xDBD8, 0x9B00]
    for t in (0x6627, 0x6628, 0xC58D, 0xC58E):
        got = mol.dropout(x[:8], t / 65536, 0)
        assert [bool(v) for v in got] == [h >= t for h in halves]


def test_dropout_of_more_than_a_launch():
    """More elements than the threads of a launch take at once, and indices past 2^31."""
    n = (1 << 31) + 100003
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = mol.dropout(x, 0.25, 99, step=2, out=x)
    for at in (0, (1 << 31) - 4000, n // 8 * 8 - 8000):
        m = min(8000, n - at)
        assert torch.equal((y[at:at + m] != 0).cpu(), rh.kept(m, 0.25, 99, 2, at))
    share = float((y.view(-1)[: 1 << 28] != 0).float().mean())
    assert abs(share - 0.75) < 5 * (0.25 * 0.75 / (1 << 28)) ** 0.5


def test_on_another_stream_and_in_a_graph():
    x, dy = rows(300, 200, BF16), rows(300, 200, BF16, seed=4)
    gamma = torch.rand(200, device="cuda") + 0.5
    step = torch.zeros(1, dtype=torch.int32, device="cuda")

    def work():
        y = mol.layer_norm(x, gamma)
        z = mol.dropout(mol.normalize(y), 0.2, 3, step=step)
        dx = mol.normalize_grad(mol.dropout(dy, 0.2, 3, step=step), y)
        return (z, dx) + mol.layer_norm_grad(dx, x, gamma)

    want = work()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = work()
    one = mol.layer_norm(x, gamma, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(one, mol.layer_norm(x, gamma))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for i in range(4):
        step.fill_(i)
        x.copy_(rows(300, 200, BF16, seed=20 + i))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, work())), f"replay {i}"
