"""Plain 64-bit forms of layer norm, the gated linear scan and 8-bit
checkpoints, each with a bound of what fp32 arithmetic may differ by.

U is half a step of fp32.  Bounds are of first order in U, per element: they
follow the formulas with every operation off by a few U.
"""
from __future__ import annotations

import torch

U = 2.0 ** -24
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}    # a rounding, relative
TINY = 2.0 ** -126


def rounded(value, bound, dtype):
    """Bound of a value rounded to `dtype` at the end."""
    return bound + STEP[dtype] * (value.abs() + bound) + TINY


def norm_forward(x, gamma, beta, eps, dtype):
    """y, its bound, mean and rstd.  A sum of C terms in a tree of at most 64
    serial additions is off by 64 U of its magnitudes' sum, so the mean is off
    by 64 U max|x|, the variance by (64 + 4) U of itself plus the mean's
    error squared, rstd by half of that."""
    x, gamma, beta = x.double(), gamma.double(), beta.double()
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    xh = (x - mean) * rstd
    y = xh * gamma + beta
    top = x.abs().amax(1, keepdim=True) * rstd
    bound = U * ((70 * top + 40 * xh.abs()) * gamma.abs() + 4 * y.abs() + 2 * beta.abs())
    return y, rounded(y, bound, dtype), mean, rstd


def norm_backward(x, mean, rstd, gamma, dy, dtype):
    """dx, dgamma, dbeta and their bounds, for x in 64 bits (or a
    checkpoint's values) and the statistics of the forward's x."""
    gamma, dy, x = gamma.double(), dy.double(), x.double()
    M, C = x.shape
    xh = (x - mean) * rstd
    a = dy * gamma
    sa, sb = a.mean(1, keepdim=True), (a * xh).mean(1, keepdim=True)
    dx = rstd * (a - sa - xh * sb)
    # xh is off by e: the mean's 70 U and rstd's 40 U (norm_forward)
    e = U * (70 * x.abs().amax(1, keepdim=True) * rstd + 44 * xh.abs())
    aa = a.abs()
    ssb = (aa * (xh.abs() * 70 * U + e)).mean(1, keepdim=True)
    bound = rstd * (U * (4 * aa + 70 * aa.mean(1, keepdim=True)) + e * sb.abs() + xh.abs() * ssb +
                    6 * U * (xh * sb).abs()) + 42 * U * dx.abs()
    # a sum over M rows: at most 64 + M / 256 additions one after another
    chain = (64 + M / 256) * U
    dgamma, dbeta = (dy * xh).sum(0), dy.sum(0)
    bg = (dy.abs() * (xh.abs() * (chain + 2 * U) + e)).sum(0) + TINY
    bb = chain * dy.abs().sum(0) + TINY
    return (dx, rounded(dx, bound, dtype)), (dgamma, bg), (dbeta, bb)


def _lengths(lengths, B, T):
    if lengths is None:
        return [T] * B
    return [min(max(int(n), 0), T) for n in lengths]


def gate(g):
    """sigmoid(g), sigmoid(-g) and the relative error of either in fp32: the
    exponent's product is off by |g| log2(e) U, so exp by |g| U + 2 U, the
    reciprocal and the product by 2 U each."""
    return torch.sigmoid(g), torch.sigmoid(-g), U * (8 + 2 * g.abs().clamp(max=100.0))


def scan_forward(g, u, reverse, lengths, h0, run=None):
    """h, hT, their bounds, and the states before each position (with bounds),
    by sweep position.  run: (states, their bounds) [B][T][I] to take before
    each 16th position instead, as the backward from checkpoints does."""
    B, T, I = g.shape
    g, u = g.double(), u.double()
    h, e = torch.zeros_like(g), torch.zeros_like(g)
    before, ebefore = torch.zeros_like(g), torch.zeros_like(g)
    hT, eT = torch.zeros((B, I), dtype=torch.float64), torch.zeros((B, I), dtype=torch.float64)
    for b, n in enumerate(_lengths(lengths, B, T)):
        v = torch.zeros(I, dtype=torch.float64) if h0 is None else h0[b].double()
        ev = torch.zeros_like(v)
        for s in range(n):
            t = n - 1 - s if reverse else s
            if run is not None and s % 16 == 0:
                v, ev = run[0][b, s], run[1][b, s]
            before[b, s], ebefore[b, s] = v, ev
            f, k, r = gate(g[b, t])
            ev = f * ev + (r + 3 * U) * ((f * v).abs() + (k * u[b, t]).abs())
            v = f * v + k * u[b, t]
            h[b, t], e[b, t] = v, ev
        hT[b], eT[b] = v, ev
    return h, e, hT, eT + TINY, before, ebefore


def scan_backward(g, u, before, ebefore, dh, reverse, lengths, dhT):
    """((dg, bound), (du, bound), (dh0, bound)), bounds before the rounding."""
    B, T, I = g.shape
    g, u, dh = g.double(), u.double(), dh.double()
    dg, du, eg, eu = (torch.zeros_like(g) for _ in range(4))
    dh0, e0 = torch.zeros((B, I), dtype=torch.float64), torch.zeros((B, I), dtype=torch.float64)
    for b, n in enumerate(_lengths(lengths, B, T)):
        G = torch.zeros(I, dtype=torch.float64) if dhT is None else dhT[b].double()
        eG = torch.zeros_like(G)
        for s in range(n - 1, -1, -1):
            t = n - 1 - s if reverse else s
            f, k, r = gate(g[b, t])
            eG = eG + U * (G.abs() + dh[b, t].abs())
            G = G + dh[b, t]
            d = before[b, s] - u[b, t]
            dg[b, t], du[b, t] = G * d * f * k, G * k
            eg[b, t] = f * k * ((eG + (2 * r + 4 * U) * G.abs()) * d.abs() + G.abs() *
                                (ebefore[b, s] + U * d.abs()))
            eu[b, t] = k * (eG + (r + U) * G.abs())
            eG = f * (eG + (r + U) * G.abs())
            G = f * G
        dh0[b], e0[b] = G, eG + TINY
    return (dg, eg), (du, eu), (dh0, e0)


def codes(x):
    """(codes, scales, values) of the 8-bit checkpoint of x, on the CPU."""
    n = x.numel()
    v = torch.nn.functional.pad(x.reshape(-1).double(), (0, -n % 64)).view(-1, 64)
    bad = ~torch.isfinite(v).all(1, keepdim=True)
    v = torch.where(bad, torch.zeros_like(v), v)
    top = v.abs().amax(1, keepdim=True)
    s = top / 127.0
    s = ((s.view(torch.int64) + (1 << 45) - 1) >> 45 << 45).view(torch.float64)   # up to 8 bits
    small = top < 2.0 ** -119
    s = torch.where(small, torch.zeros_like(s), s)
    q = torch.where(small, torch.zeros_like(v), torch.round(v / torch.where(small, torch.ones_like(s), s)))
    scale = torch.where(bad, torch.full_like(s, float("nan")), s)
    return (q.reshape(-1)[:n].view(x.shape).to(torch.int8), scale.reshape(-1).to(torch.bfloat16),
            (q * scale).reshape(-1)[:n].view(x.shape))
