"""Plain float64 forms of the operators that learn the similarity, with
bounds on what float32 arithmetic may add to each of their outputs.

U is half a unit in the last place of float32 (a rounding's largest relative
error).  A sum of n terms in any order is off by at most (n - 1) U times the
sum of their magnitudes (first order), whatever tree it is formed in."""
from __future__ import annotations

import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # largest relative error of one rounding


def within(got, want, bound, what):
    """|got - want| <= bound elementwise (float64; NaN and infinities in the same places)."""
    got, want = got.double().cpu(), want.double().cpu()
    bound = torch.as_tensor(bound, dtype=torch.float64).cpu().expand_as(want)
    assert got.shape == want.shape, what
    assert bool((torch.isnan(got) == torch.isnan(want)).all()), f"{what}: NaN in other places"
    err = torch.where(torch.isnan(want) | (got == want), 0.0, (got - want).abs())
    bad = err > bound
    if bool(bad.any()):
        i = int(torch.argmax(torch.where(bad, err / bound.clamp(min=1e-300), 0.0)))
        raise AssertionError(f"{what}: {int(bad.sum())} of {err.numel()} off, worst at {i}: got {got.flatten()[i].item()}, "
                             f"want {want.flatten()[i].item()}, bound {bound.flatten()[i].item()}")


def embed_grad(grad, ids, V, scale):
    """(sums, bounds): rows of grad [C][T][d] summed by id; a row of n tokens takes n additions and one product."""
    C, T, d = grad.shape
    g = grad.double().cpu()
    ids = ids.cpu().long()
    ok = (ids >= 0) & (ids < V)
    out, mag, n = torch.zeros(C, V, d, dtype=torch.float64), torch.zeros(C, V, d, dtype=torch.float64), torch.zeros(V)
    out.index_add_(1, ids[ok], g[:, ok])
    mag.index_add_(1, ids[ok], g[:, ok].abs())
    n.index_add_(0, ids[ok], torch.ones(int(ok.sum())))
    return out * scale, mag * abs(scale) * ((n + 2) * U)[None, :, None]


def softmax_loss(phi, target, ids, inv_temp, weight):
    """(loss, dphi, loss bound, dphi bound)."""
    phi, target = phi.double().cpu(), target.cpu().long()
    B, N = phi.shape
    keep = torch.ones(B, N, dtype=torch.bool)
    dead = (target < 0) | (target >= N)
    t = target.clamp(0, N - 1)
    rows = torch.arange(B)
    if ids is not None:
        ids = ids.cpu().long()
        dead |= ids[t] < 0
        keep &= (ids >= 0)[None] & (ids[None] != ids[t][:, None])
        keep[rows, t] = True
    z = torch.where(keep, phi * inv_temp, -torch.inf)
    m = z.amax(1, keepdim=True)
    e = torch.where(keep, torch.exp(z - m), 0.0)
    s = e.sum(1, keepdim=True)
    zt = phi[rows, t] * inv_temp
    loss = torch.log(s[:, 0]) + m[:, 0] - zt
    w = (torch.ones(B, dtype=torch.float64) if weight is None else weight.double().cpu()) * inv_temp
    p = e / s
    hot = torch.zeros(B, N, dtype=torch.float64)
    hot[rows, t] = 1.0
    dphi = torch.where(keep, w[:, None] * (p - hot), 0.0)
    # z and z - m: 3 roundings of at most the row's largest |z|; the exponential
    # 8 U of itself; sums of at most 32 values in a thread, then trees of at
    # most 10 + 4 levels (longer rows: 40 parts of them)
    big = torch.where(keep & torch.isfinite(z), z.abs(), 0.0).amax(1)
    rel = U * (4 * big + 8 + 64 + N / 1024 + 40)
    loss_b = rel + U * 4 * (m[:, 0].abs() + zt.abs() + loss.abs())
    # an exponential below float32's smallest normal number may come out as 0:
    # the probability, at most it (the sum is 1 or more), is off by at most 2^-126
    dphi_b = w.abs()[:, None] * (p * (2 * rel[:, None] + 8 * U) + hot * 4 * U + 2.0 ** -126) + 1e-45
    loss, dphi = loss.masked_fill(dead, 0.0), dphi.masked_fill(dead[:, None], 0.0)
    return loss, dphi, loss_b, dphi_b


def score_grads(inputs, dphi):
    """({name: gradient}, {name: bound}) of sum(dphi * phi) for the tensors
    (Q, X, a_q, a_x, W1, b1, W2, b2), from the formulas, with the bound that
    follows the roundings of a float32 evaluation through the chain to first
    order (doubled for what second order adds)."""
    dt = inputs[0].dtype
    Q, X, a_q, a_x, W1, b1, W2, b2 = (t.double().cpu() for t in inputs)
    g = dphi.double().cpu()
    (B, Pq, d), (Px, N, _), (H, P) = Q.shape, X.shape, W1.shape
    s = torch.einsum("bqd,xnd->bnqx", Q, X).reshape(B, N, P)
    es = (d + 1) * U * torch.einsum("bqd,xnd->bnqx", Q.abs(), X.abs()).reshape(B, N, P)
    u = s @ W1.t() + b1
    eu = es @ W1.abs().t() + (P + 2) * U * (s.abs() @ W1.abs().t() + b1.abs())
    sig = torch.sigmoid(u)
    h = u * sig
    eh = 1.1 * eu + 6 * U * h.abs()                      # |SiLU'| <= 1.1
    lg = a_q[:, None] + a_x[None] + b2 + h @ W2.t()
    el = eh @ W2.abs().t() + (H + 4) * U * (h.abs() @ W2.abs().t() + a_q.abs()[:, None] + a_x.abs()[None] + b2.abs())
    pi = torch.softmax(lg, -1)
    # softmax: the exponent's error, its rounding and the sum's
    rpi = 2 * el.amax(-1, keepdim=True) + U * (2 * (lg - lg.amax(-1, keepdim=True)).abs() + P + 12)
    phi = (pi * s).sum(-1, keepdim=True)
    ephi = (pi * (es + s.abs() * (rpi + (P + 4) * U))).sum(-1, keepdim=True)
    gpi = g[..., None] * pi
    egpi = gpi.abs() * (rpi + 4 * U)
    dl = gpi * (s - phi)
    edl = egpi * (s.abs() + phi.abs()) + gpi.abs() * (es + ephi + 3 * U * (s.abs() + phi.abs()))
    dh = dl @ W2
    edh = edl @ W2.abs() + (P + 1) * U * (dl.abs() @ W2.abs())
    k = sig * (1 + u * (1 - sig))
    du = dh * k
    edu = 1.1 * edh + dh.abs() * (0.5 * eu + 8 * U * (1 + u.abs()))   # |SiLU''| <= 0.5
    ds = gpi + du @ W1
    eds = egpi + edu @ W1.abs() + (H + 2) * U * (gpi.abs() + du.abs() @ W1.abs())

    def total(x, ex, dims, n):                           # a sum over pairs
        return x.sum(dims), ex.sum(dims) + n * U * x.abs().sum(dims)

    def product(a, ea, b, eb):                           # sum over pairs of a b^T
        f = (lambda x: x.reshape(B * N, -1))
        a, ea, b, eb = f(a), f(ea), f(b), f(eb)
        return a.t() @ b, ea.t() @ b.abs() + a.abs().t() @ eb + (B * N + 2) * U * (a.abs().t() @ b.abs())

    out, bound = {}, {}
    out["da_q"], bound["da_q"] = total(dl, edl, 1, N)
    out["da_x"], bound["da_x"] = total(dl, edl, 0, B)
    out["db2"], bound["db2"] = total(dl, edl, (0, 1), B * N)
    out["db1"], bound["db1"] = total(du, edu, (0, 1), B * N)
    out["dW1"], bound["dW1"] = product(du, edu, s, es)
    out["dW2"], bound["dW2"] = product(dl, edl, h, eh)
    ds5, ds5a = ds.view(B, N, Pq, Px), ds.view(B, N, Pq, Px).abs()
    e5 = eds.view(B, N, Pq, Px) + (2.0 ** -16 * ds5a if dt == torch.bfloat16 else 0.0)   # two bf16 terms
    out["dQ"] = torch.einsum("bnqx,xnd->bqd", ds5, X)
    bound["dQ"] = torch.einsum("bnqx,xnd->bqd", e5 + N * Px * U * ds5a, X.abs())
    out["dX"] = torch.einsum("bnqx,bqd->xnd", ds5, Q)
    bound["dX"] = torch.einsum("bnqx,bqd->xnd", e5 + B * Pq * U * ds5a, Q.abs())
    for name in out:
        half = HALF[dt] if name in ("dQ", "dX", "dW1", "dW2") else U
        bound[name] = 2 * bound[name] + half * (1 + 2 * half) * out[name].abs() + 1e-40
    return out, bound


def mol_inputs(B, N, Pq, Px, d, H, dtype, seed, std=0.3, device="cpu"):
    """(Q, X, a_q, a_x, W1, b1, W2, b2) and dphi, drawn on the CPU."""
    gen = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    unit = lambda v: v / v.norm(dim=-1, keepdim=True)  # noqa: E731
    P = Pq * Px
    t = [unit(randn(B, Pq, d)).to(dtype), unit(randn(Px, N, d)).to(dtype), std * randn(B, P), std * randn(N, P),
         (std * randn(H, P)).to(dtype), std * randn(H), (std * randn(P, H)).to(dtype), std * randn(P)]
    g = torch.softmax(2 * randn(B, N), 1)
    g[torch.arange(B), torch.randint(0, N, (B,), generator=gen)] -= 1.0
    return [x.to(device) for x in t], (g / B).to(device)


def adamw(p, g, m, v, lr, beta1, beta2, eps, decay, step, scale=1.0):
    """(p', m', v') in float64."""
    p, g, m, v = (t.double().cpu() for t in (p, g, m, v))
    g = g * scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    return p * (1 - lr * decay) - lr * (m / (1 - beta1 ** step)) / ((v / (1 - beta2 ** step)).sqrt() + eps), m, v
