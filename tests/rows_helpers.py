"""Plain float64 forms of the operators between embedding rows and scores, with
bounds on what float32 arithmetic may add to each output.

U is half a unit in the last place of float32.  A sum over a row is formed by at
most 16 additions in a lane, 6 over a wave's lanes and 15 over waves: every term
passes at most PATH roundings."""
from __future__ import annotations

import numpy as np
import torch

from learn_helpers import HALF, U

PATH = 40


def _norm_parts(x, eps):
    """(xhat, its bound, rstd, rstd's relative bound)"""
    x = x.double().cpu()
    d = x.shape[-1]
    mean = x.mean(-1, keepdim=True)
    c = x - mean
    var = (c * c).mean(-1, keepdim=True)
    rstd = 1.0 / (var + eps).sqrt()
    dm = (PATH + 1) * U * x.abs().mean(-1, keepdim=True)            # the mean's error
    dc = dm + U * c.abs()
    # the sum of squares: 2 c dc a term, and its own roundings; var + eps, the root, the quotient: 4 more
    dvar = (2 * c.abs() * dc).mean(-1, keepdim=True) + dm * dm + (PATH + 2) * U * var
    rel = 0.5 * dvar / (var + eps) + 4 * U
    return c * rstd, dc * rstd + (c * rstd).abs() * (rel + U), rstd, rel, d


def layer_norm(x, gamma, beta, eps, out):
    """(y, bound)"""
    xhat, dxhat, _, _, d = _norm_parts(x, eps)
    g = torch.ones(d, dtype=torch.float64) if gamma is None else gamma.double().cpu()
    b = torch.zeros(d, dtype=torch.float64) if beta is None else beta.double().cpu()
    y = xhat * g + b
    return y, dxhat * g.abs() + 2 * U * ((xhat * g).abs() + b.abs()) + HALF[out] * y.abs() * 1.01


def layer_norm_grad(dy, x, gamma, eps, out):
    """(dx, dgamma, dbeta) and their bounds"""
    xhat, dxhat, rstd, rel, d = _norm_parts(x, eps)
    dy = dy.double().cpu()
    w = dy if gamma is None else dy * gamma.double().cpu()
    c1, c2 = w.mean(-1, keepdim=True), (w * xhat).mean(-1, keepdim=True)
    dc1 = (PATH + 3) * U * w.abs().mean(-1, keepdim=True)
    dc2 = ((PATH + 4) * U * (w * xhat).abs() + w.abs() * dxhat).mean(-1, keepdim=True)
    dx = rstd * (w - c1 - xhat * c2)
    size = w.abs() + c1.abs() + (xhat * c2).abs()
    bound = rstd * (U * w.abs() + dc1 + xhat.abs() * dc2 + c2.abs() * dxhat + 4 * U * size + rel * size)
    flat, fx, fd = dy.reshape(-1, d), xhat.reshape(-1, d), dxhat.reshape(-1, d)
    # a lane's rows (5 of 5000 at most), 6 over lanes, 3 over waves, 80 over workgroups
    dgamma, dbeta = (flat * fx).sum(0), flat.sum(0)
    bg = (flat.abs() * fd).sum(0) + 128 * U * (flat * fx).abs().sum(0)
    return (dx, dgamma, dbeta), (bound + HALF[out] * dx.abs() * 1.01, bg, 128 * U * flat.abs().sum(0))


def normalize(x, eps, out):
    x = x.double().cpu()
    r = x.square().sum(-1, keepdim=True).sqrt()
    y = x / r.clamp(min=eps)
    return y, (PATH + 10) * U * y.abs() + HALF[out] * y.abs() * 1.01


def normalize_grad(dy, x, eps, out):
    x, dy = x.double().cpu(), dy.double().cpu()
    r = x.square().sum(-1, keepdim=True).sqrt()
    size = r.clamp(min=eps)
    y = x / size
    along = torch.where(r > eps, (y * dy).sum(-1, keepdim=True), 0.0)
    dx = (dy - y * along) / size
    mag = (y * dy).abs().sum(-1, keepdim=True)
    # y is off by PATH / 2 + 6 roundings, the product's sum by PATH + 1 more, the quotient by as much as y
    bound = ((PATH + 10) * U * dy.abs() + y.abs() * (3 * PATH + 30) * U * mag) / size
    return dx, bound + HALF[out] * dx.abs() * 1.01


# ------------------------------------------------------------------ dropout
def philox(counter, key, rounds=10):
    """Philox 4x32 (Salmon et al. 2011) of counters [..., 4] under one key: uint32 [..., 4]."""
    c = [np.asarray(counter[..., i], dtype=np.uint64) for i in range(4)]
    k = [np.uint64(key[0]), np.uint64(key[1])]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & low, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + np.uint64(0x9E3779B9)) & low, (k[1] + np.uint64(0xBB67AE85)) & low]
    return np.stack(c, axis=-1).astype(np.uint32)


def kept(n, p, seed, step, offset):
    """Which of n elements dropout keeps."""
    blocks = (n + 7) // 8
    at = np.arange(blocks, dtype=np.uint64) + np.uint64(offset // 8)
    counter = np.stack([at & np.uint64(0xFFFFFFFF), at >> np.uint64(32), np.full(blocks, step, np.uint64),
                        np.zeros(blocks, np.uint64)], axis=-1)
    words = philox(counter, (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF))
    halves = np.stack([words & 0xFFFF, words >> 16], axis=-1).reshape(-1)[:n]
    return torch.from_numpy(halves >= int(np.floor(p * 65536 + 0.5)))


def dropout(x, p, seed, step, offset, residual, out):
    keep = kept(x.numel(), p, seed, step, offset).view(x.shape)
    t = int(np.floor(p * 65536 + 0.5))
    y = torch.where(keep, x.double().cpu() * (65536.0 / (65536 - t)), 0.0)
    bound = 3 * U * y.abs()                                    # the factor, the product, the sum
    if residual is not None:
        y = y + residual.double().cpu()
        bound = bound + U * y.abs()
    return keep, y, bound + HALF[out] * y.abs() * 1.01


# ------------------------------------------------------------------ the gated scan
STEP = 16      # roundings a token adds to the state: the gate's 11 (e^-|g| 4, 1 + e, the quotient, the product), three products and sums
JOIN = 64      # and those of joining slices, waves, chunks and groups on the way to it
# Below 2^-126 a float32 rounding is off by up to 2^-126 whatever the value (it may be flushed to 0), not by a share of it:
# T tokens' STEP roundings, none of which grows on its way (f <= 1), are off by up to STEP T 2^-126 together.
TINY = 2.0 ** -126


def _gates(gate):
    g = gate.double().cpu()
    return torch.sigmoid(g), torch.sigmoid(-g)


def gated_scan(gate, x, lens, first, h0, out):
    """(h, bound, live rows, last, last's bound) of histories of these lengths, packed from row ``first`` on."""
    f, r = _gates(gate)
    x = x.double().cpu()
    T, d = x.shape
    h, hb, err = (torch.zeros(T, d, dtype=torch.float64) for _ in range(3))
    live = torch.zeros(T, dtype=torch.bool)
    last, lb = torch.zeros(len(lens), d, dtype=torch.float64), torch.zeros(len(lens), d, dtype=torch.float64)
    t = first
    for b, n in enumerate(lens):
        s = torch.zeros(d, dtype=torch.float64) if h0 is None else h0[b].double().cpu()
        sb, e = s.abs(), torch.zeros(d, dtype=torch.float64)
        live[t:t + n] = True
        for t in range(t, t + n):
            s = f[t] * s + r[t] * x[t]
            sb = f[t] * sb + r[t] * x[t].abs()
            e = f[t] * e + STEP * U * sb
            h[t], hb[t], err[t] = s, sb, e
        t = t + 1 if n else t
        last[b], lb[b] = s, e + (JOIN * U * sb if n else 0.0)
    tiny = STEP * T * TINY
    return h, err + JOIN * U * hb + HALF[out] * h.abs() * 1.01 + tiny, live, last, lb + tiny


def gated_scan_grad(gate, x, h, dh, lens, first, h0, dlast, out):
    """((dgate, bound), (dx, bound), (dh0, bound))"""
    f, r = _gates(gate)
    x, h = x.double().cpu(), h.double().cpu()
    T, d = x.shape
    B = len(lens)
    dh = torch.zeros(T, d, dtype=torch.float64) if dh is None else dh.double().cpu()
    D, Db, err = (torch.zeros(T, d, dtype=torch.float64) for _ in range(3))
    prev = torch.zeros(T, d, dtype=torch.float64)
    dh0, b0 = torch.zeros(B, d, dtype=torch.float64), torch.zeros(B, d, dtype=torch.float64)
    start = first
    for b, n in enumerate(lens):
        E = torch.zeros(d, dtype=torch.float64) if dlast is None else dlast[b].double().cpu()
        Eb, e = E.abs(), torch.zeros(d, dtype=torch.float64)
        for t in range(start + n - 1, start - 1, -1):
            D[t], Db[t] = dh[t] + E, dh[t].abs() + Eb
            err[t] = e + STEP * U * Db[t]
            prev[t] = h[t - 1] if t > start else (0.0 if h0 is None else h0[b].double().cpu())
            E, Eb, e = f[t] * D[t], f[t] * Db[t], f[t] * err[t]
        dh0[b], b0[b] = E, e + ((STEP + JOIN) * U * Eb if n else 0.0)
        start += n
    err = err + JOIN * U * Db
    k = f * r * (prev - x)
    dgate, dx = k * D, r * D
    # (as above; dgate's factors, f (1 - f) and the difference, can be up to |prev - x| / 4)
    tiny = STEP * T * TINY
    bg = k.abs() * (err + 32 * U * Db) + HALF[out] * dgate.abs() * 1.01 + tiny * (1 + (prev - x).abs())
    bx = r * (err + STEP * U * Db) + HALF[out] * dx.abs() * 1.01 + tiny
    return (dgate, bg), (dx, bx), (dh0, b0 + tiny)
