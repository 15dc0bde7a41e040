"""The gated scan where states are not finite, in packed sets that its long slices
cut, and past the caches (MI355X only)."""
import itertools

import pytest
import torch

import rows_helpers as rh
from learn_helpers import within
from paper_2407_15462_amd import mol
from parity_helpers import log
from test_gpu_rows import fenced, off_by_one, unharmed
from test_gpu_scan import make

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
NAME = {F32: "f32", BF16: "bf16"}
INF, NAN = float("inf"), float("nan")


def same(a, b):
    return torch.equal(a, b)


def holds(t, value):
    return bool((torch.isnan(t) if value != value else t == value).all())


# The middle history is the poisoned one: within one slice and chunk, over several groups of chunks, and over several
# supers; of 40,000 tokens x 130 bfloat16 channels the scan takes slices of 32 tokens.
@pytest.mark.parametrize("n,at", [(90, 10), (4096, 10), (4096, 2999), (40000, 17000)])
@pytest.mark.parametrize("d,t", [(3, F32), (8, BF16), (64, BF16), (130, BF16), (130, F32), (201, BF16)])
@pytest.mark.parametrize("level", [0.0, 2.0, -30.0])
def test_what_is_not_finite_stays_to_the_end(n, at, d, t, level):
    """h_t = f_t h_{t-1} + (1 - f_t) x_t with f_t > 0: a NaN or an infinity stays in a history's states for good (back: in
    all that lies before it), also where the product of the gates since is below float32's range; and in no other's."""
    log(f"[scan] not finite: n={n} at={at} d={d} {NAME[t]} gates {level}")
    lens = [70, n, 40]
    T, lo = sum(lens), lens[0]
    hi = lo + n
    g = torch.Generator(device="cuda").manual_seed(n + d)
    gate = torch.full((T, d), level, dtype=t, device="cuda")
    x = torch.rand(T, d, generator=g, device="cuda").to(t)
    dh = (1 + torch.rand(T, d, generator=g, device="cuda")).to(t)
    h0, dlast = torch.rand(3, d, generator=g, device="cuda"), torch.rand(3, d, generator=g, device="cuda")
    offsets = torch.tensor(list(itertools.accumulate([0] + lens)), dtype=torch.int32, device="cuda")
    clean, end = mol.gated_scan(gate, x, offsets, h0=h0)
    cg = mol.gated_scan_grad(gate, x, clean, dh=dh, offsets=offsets, h0=h0, dlast=dlast)
    assert torch.isfinite(clean).all() and all(torch.isfinite(a).all() for a in cg)
    for value in (NAN, INF, -INF):
        bad = x.clone()
        bad[lo + at] = value
        h, last = mol.gated_scan(gate, bad, offsets, h0=h0)
        assert same(h[:lo + at], clean[:lo + at]) and same(h[hi:], clean[hi:]) and same(last[[0, 2]], end[[0, 2]])
        assert holds(h[lo + at:hi], value) and holds(last[1], value), f"x = {value}"
        start = h0.clone()
        start[1] = value
        h, last = mol.gated_scan(gate, x, offsets, h0=start)
        assert same(h[:lo], clean[:lo]) and same(h[hi:], clean[hi:]) and same(last[[0, 2]], end[[0, 2]])
        assert holds(h[lo:hi], value) and holds(last[1], value), f"h0 = {value}"
        bad = dh.clone()
        bad[lo + at] = value
        dg, dx, d0 = mol.gated_scan_grad(gate, x, clean, dh=bad, offsets=offsets, h0=h0, dlast=dlast)
        for p, q in ((dg, cg[0]), (dx, cg[1])):
            assert same(p[:lo], q[:lo]) and same(p[lo + at + 1:], q[lo + at + 1:])
        assert same(d0[[0, 2]], cg[2][[0, 2]])
        assert holds(dx[lo:lo + at + 1], value) and holds(d0[1], value), f"dh = {value}"
        assert not torch.isfinite(dg[lo:lo + at + 1]).any()
        bad = dlast.clone()
        bad[1] = value
        dg, dx, d0 = mol.gated_scan_grad(gate, x, clean, dh=dh, offsets=offsets, h0=h0, dlast=bad)
        for p, q in ((dg, cg[0]), (dx, cg[1])):
            assert same(p[:lo], q[:lo]) and same(p[hi:], q[hi:])
        assert holds(dx[lo:hi], value) and holds(d0[1], value), f"dlast = {value}"
    # a NaN gate: every state from its token on
    bad = gate.clone()
    bad[lo + at] = NAN
    h, last = mol.gated_scan(bad, x, offsets, h0=h0)
    assert same(h[:lo + at], clean[:lo + at]) and same(h[hi:], clean[hi:]) and same(last[[0, 2]], end[[0, 2]])
    assert holds(h[lo + at:hi], NAN) and holds(last[1], NAN)


def packed(T, seed):
    """(lengths, rows in front, rows behind) of about T tokens: histories of no token to several chunks."""
    g = torch.Generator().manual_seed(seed)
    pool = [0, 1, 2, 3, 31, 32, 33, 63, 64, 65, 255, 256, 257, 700]
    lens = [0, 0, 1]
    while sum(lens) < T:
        lens.append(pool[int(torch.randint(0, len(pool), (1,), generator=g))])
    lens += [0]
    return lens, 37, 45


@pytest.mark.parametrize("d", [130, 131])
@pytest.mark.parametrize("to", [F32, BF16])
def test_packed_histories_in_long_slices(d, to):
    """bfloat16 histories of more than 256 units, which the scan takes in slices of 32 tokens: several beginnings and
    ends in one, and both sides of every cut."""
    lens, front, back = packed(36000, seed=d)
    T = front + sum(lens) + back
    assert T > 128 * 256, "two groups of channels: 256 units"
    log(f"[scan] packed: {len(lens)} histories of {T} tokens x {d} -> {NAME[to]}")
    gate, x, offsets, h0, dead = make(lens, front, back, d, BF16)
    live, on = ~dead, (~dead).cuda()
    for start in (h0, None):
        want, bound, _, last, lb = rh.gated_scan(gate, x, lens, front, start, to)
        out, buf = fenced((T, d), to)
        end, ebuf = fenced((len(lens), d), F32)
        mol.gated_scan(gate, x, offsets, h0=start, out=out, last=end)
        within(out[on], want[live], bound[live], "h")
        within(end, last, lb, "last")
        assert unharmed(buf, T * d) and unharmed(ebuf, len(lens) * d) and bool((out[~on] == 77).all())
        h, e = mol.gated_scan(off_by_one(gate), off_by_one(x), offsets, h0=start, dtype=to)
        assert torch.equal(h[on], out[on]) and torch.equal(e, end), "unaligned rows or a second run differ"
    g = torch.Generator().manual_seed(d)
    dh = torch.randn(T, d, generator=g).to(to).cuda()
    dh[~on] = float("nan")
    dlast = torch.randn(len(lens), d, generator=g).cuda()
    ref = rh.gated_scan_grad(gate, x, out, dh, lens, front, None, dlast, BF16)
    got = mol.gated_scan_grad(gate, x, out, dh=dh, offsets=offsets, dlast=dlast)
    for name, a, b in zip(("dgate", "dx"), got, ref):
        within(a[on], b[0][live], b[1][live], name)
        assert not a[~on].any()


def test_float32_scan_past_the_caches():
    """256 MB and more of float32 rows: some histories against float64, and as they are alone."""
    d, n, B = 512, 700, 101
    T = n * B
    assert T * d * 8 >= 1 << 28
    g = torch.Generator(device="cuda").manual_seed(6)
    gate, x, dh = (torch.randn(T, d, generator=g, device="cuda") for _ in range(3))
    gate += 2
    offsets = torch.arange(B + 1, dtype=torch.int32, device="cuda") * n
    h, last = mol.gated_scan(gate, x, offsets)
    dg, dx, _ = mol.gated_scan_grad(gate, x, h, dh=dh, offsets=offsets)
    for b in (0, 50, 100):
        rows = slice(b * n, b * n + n)
        gb, xb, hb, db = (t[rows].contiguous() for t in (gate, x, h, dh))
        want, bound, _, end, lb = rh.gated_scan(gb, xb, [n], 0, None, F32)
        within(hb, want, bound, f"h of history {b}")
        within(last[b:b + 1], end, lb, f"last of history {b}")
        ref = rh.gated_scan_grad(gb, xb, hb, db, [n], 0, None, None, F32)
        within(dg[rows], *ref[0], f"dgate of history {b}")
        within(dx[rows], *ref[1], f"dx of history {b}")
