"""The gated scan where states are not finite (MI355X only)."""
import itertools

import pytest
import torch

from paper_2407_15462_amd import mol
from parity_helpers import log

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
