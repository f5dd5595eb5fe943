"""Plain 64-bit forms of the causal convolution, the selective scan, group norm with an
activation and AdamW with moments in 32 or 8 bits, each with a bound of what fp32
arithmetic may differ by.

U is half a step of fp32.  Bounds are of first order in U, per element: an operation is off by U of its result
(2 U where the hardware's exponential, logarithm or reciprocal is off by a step), a sum of n
terms one after another by n U of their magnitudes' sum.
"""
from __future__ import annotations

import torch

from tests.seq_ref import TINY, U, rounded

F64 = torch.float64


def lengths_of(lengths, B, T):
    return [T] * B if lengths is None else [min(max(int(n), 0), T) for n in lengths]


def sweep(v, ns, reverse):
    """[B][T][..] by sweep position, 0 past each length (its own inverse)."""
    out = torch.zeros_like(v, dtype=F64)
    for b, n in enumerate(ns):
        row = v[b, :n].to(F64)
        out[b, :n] = row.flip(0) if reverse else row
    return out


def act_of(v, ev, act):
    """act(v), its slope, and their errors for an argument off by ev.  sigmoid is off by
    (8 + 2 |v|) U of itself (its exponent by |v| log2(e) U), slopes of silu are at most 1.1 and those
    of its slope 0.5."""
    if act == "none":
        return v, torch.ones_like(v), ev, torch.zeros_like(v)
    s = torch.sigmoid(v)
    slope = s * (1 + v * (1 - s))
    r = U * (8 + 2 * v.abs().clamp(max=100.0))
    return v * s, slope, 1.1 * ev + r * (v * s).abs(), 0.5 * ev + r * s * (2 + 2 * v.abs() * (1 - s))


# ------------------------------------------------------------------ convolution

def conv_forward(x, w, bias, act, reverse, lengths, state):
    """a [B][T][I] by position (with its error), y by step with its bound before rounding, the state after, padded inputs."""
    B, T, I = x.shape
    K = w.shape[1]
    ns = lengths_of(lengths, B, T)
    before = torch.zeros((B, K - 1, I), dtype=F64) if state is None else state.to(F64)
    xs = torch.cat([before, sweep(x, ns, reverse)], 1)
    w, bias = w.to(F64), torch.zeros(I, dtype=F64) if bias is None else bias.to(F64)
    a, mag = bias.expand(B, T, I).clone(), bias.abs().expand(B, T, I).clone()
    for k in range(K):
        a = a + w[:, k] * xs[:, k:k + T]
        mag = mag + (w[:, k] * xs[:, k:k + T]).abs()
    ea = (K + 1) * U * mag
    y, _, ey, _ = act_of(a, ea, act)
    live = torch.tensor([[s < n for s in range(T)] for n in ns])[:, :, None]
    after = torch.stack([xs[b, n:n + K - 1] for b, n in enumerate(ns)])
    return (sweep(y * live, ns, reverse), sweep(ey * live, ns, reverse)), after, (a, ea, xs, live, ns)


def conv_backward(kept, w, dy, act, reverse, dstate_out):
    a, ea, xs, live, ns = kept
    B, T, I = a.shape
    K = w.shape[1]
    w = w.to(F64)
    g = sweep(dy, ns, reverse)
    _, slope, _, es = act_of(a, ea, act)
    da, eda = g * slope * live, g.abs() * (es + 2 * U * slope.abs()) * live
    dxs, edx = torch.zeros_like(xs), torch.zeros_like(xs)
    dw, edw = torch.zeros_like(w), torch.zeros_like(w)
    chain = (B * T + 8) * U
    for k in range(K):
        dxs[:, k:k + T] += w[:, k] * da
        edx[:, k:k + T] += w[:, k].abs() * (eda + (K + 1) * U * da.abs())
        dw[:, k] = (da * xs[:, k:k + T]).sum((0, 1))
        edw[:, k] = (xs[:, k:k + T].abs() * (eda + chain * da.abs())).sum((0, 1))
    if dstate_out is not None:
        for b, n in enumerate(ns):
            dxs[b, n:n + K - 1] += dstate_out[b].to(F64)
            edx[b, n:n + K - 1] += U * dstate_out[b].to(F64).abs() + U * dxs[b, n:n + K - 1].abs()
    db, edb = da.sum((0, 1)), (eda + chain * da.abs()).sum((0, 1))
    return ((sweep(dxs[:, K - 1:], ns, reverse), sweep(edx[:, K - 1:], ns, reverse)), (dw, edw + TINY), (db, edb + TINY),
            (dxs[:, :K - 1], edx[:, :K - 1] + TINY))


# --------------------------------------------------------------- selective scan

class Select:
    """The scan in 64 bits by sweep position.  Errors: d = softplus(raw), off by what raw is (U |raw|, slope
    sigmoid) and by (14 + 2 |raw|) U of itself; a decay exp(d A) by |A| ed and (16 |d A| + 6) U of itself (its exponent is a product of
    rounded numbers, and runs of 8 steps are also folded by the exponential of their sum); a state by a few U
    for each of the folds that it passes."""

    def __init__(self, u, delta, A, Bm, Cm, D=None, z=None, dbias=None, softplus=False, reverse=False, lengths=None, h0=None):
        B, T, I = u.shape
        S = A.shape[1]
        self.B, self.T, self.I, self.S, self.reverse, self.softplus = B, T, I, S, reverse, softplus
        self.ns = ns = lengths_of(lengths, B, T)
        self.live = torch.tensor([[s < n for s in range(T)] for n in ns])[:, :, None]
        zero = torch.zeros(I, dtype=F64)
        self.A, self.D = A.to(F64), zero if D is None else D.to(F64)
        self.u, self.Bm, self.Cm = (sweep(v, ns, reverse) for v in (u, Bm, Cm))
        self.z = None if z is None else sweep(z, ns, reverse)
        self.raw = sweep(delta, ns, reverse) + (zero if dbias is None else dbias.to(F64))
        eraw = U * self.raw.abs()
        if softplus:
            self.d = torch.nn.functional.softplus(self.raw, threshold=1e9)
            self.ed = eraw * torch.sigmoid(self.raw) + U * (14 + 2 * self.raw.abs().clamp(max=100.0)) * self.d
        else:
            self.d, self.ed = self.raw, eraw
        self.d, self.ed = self.d * self.live, self.ed * self.live
        du, edu = self.d * self.u, (self.ed + U * self.d.abs()) * self.u.abs()
        self.du, self.edu = du, edu
        h = torch.zeros((B, I, S), dtype=F64) if h0 is None else h0.to(F64)
        eh = torch.zeros_like(h)
        self.hs, self.ehs, self.a, self.ra = [h], [eh], [], []
        for s in range(T):
            x = self.d[:, s, :, None] * self.A
            a = torch.exp(x)
            ra = self.ed[:, s, :, None] * self.A.abs() + U * (16 * x.abs() + 6)
            b = du[:, s, :, None] * self.Bm[:, s, None]
            eb = (edu[:, s, :, None] + 2 * U * du[:, s, :, None].abs()) * self.Bm[:, s, None].abs()
            eh = a * eh + (ra + 3 * U) * (a * h).abs() + eb + 3 * U * b.abs()
            h = a * h + b
            self.hs.append(h)
            self.ehs.append(eh)
            self.a.append(a)
            self.ra.append(ra)
        C = self.Cm[:, :, None]
        H, EH = torch.stack(self.hs[1:], 1), torch.stack(self.ehs[1:], 1)
        self.p = (H * C).sum(-1) + self.D * self.u
        self.ep = (C.abs() * (EH + (S + 6) * U * H.abs())).sum(-1) + 3 * U * (self.D * self.u).abs()
        if z is None:
            y, ey = self.p, self.ep
        else:
            g, _, eg, _ = act_of(self.z, torch.zeros_like(self.z), "silu")
            y, ey = self.p * g, self.ep * g.abs() + self.p.abs() * (eg + U * g.abs())
        self.y, self.ey = sweep(y * self.live, ns, reverse), sweep(ey * self.live, ns, reverse)
        self.hT, self.ehT = h, eh + TINY

    def backward(self, dy, dhT=None):
        """{name: (value, bound before rounding)}"""
        B, T, I, S, live = self.B, self.T, self.I, self.S, self.live
        g = sweep(dy, self.ns, self.reverse)
        dp, edp = g, torch.zeros_like(g)
        out = {}
        if self.z is not None:
            v, slope, ev, es = act_of(self.z, torch.zeros_like(self.z), "silu")
            dp, edp = g * v, g.abs() * (ev + U * v.abs())
            dz = g * self.p * slope
            out["dz"] = (dz, g.abs() * (self.ep * slope.abs() + self.p.abs() * (es + 3 * U * slope.abs())))
        dp, edp = dp * live, edp * live
        G = torch.zeros((B, I, S), dtype=F64) if dhT is None else dhT.to(F64)
        eG = torch.zeros_like(G)
        q, eq, w, ew = (torch.zeros((B, T, I), dtype=F64) for _ in range(4))
        dB, eB, dC, eC = (torch.zeros((B, T, S), dtype=F64) for _ in range(4))
        dA, eA = torch.zeros((I, S), dtype=F64), torch.zeros((I, S), dtype=F64)
        lanes, steps, terms = 24 + I // 16, B * T + 16, S + 6       # additions one after another
        for s in range(T - 1, -1, -1):
            C, Bm = self.Cm[:, s, None], self.Bm[:, s, None]
            c = C * dp[:, s, :, None]
            eG = eG + C.abs() * edp[:, s, :, None] + 2 * U * (c.abs() + G.abs())
            G = G + c
            h, eh = self.hs[s + 1], self.ehs[s + 1] + 2 * U * self.hs[s + 1].abs()
            x = dp[:, s, :, None]
            dC[:, s] = (h * x).sum(1)
            eC[:, s] = (eh * x.abs() + h.abs() * (edp[:, s, :, None] + lanes * U * x.abs())).sum(1)
            x = self.du[:, s, :, None]
            dB[:, s] = (G * x).sum(1)
            eB[:, s] = (eG * x.abs() + G.abs() * (self.edu[:, s, :, None] + lanes * U * x.abs())).sum(1)
            q[:, s], eq[:, s] = (G * Bm).sum(-1), (Bm.abs() * (eG + terms * U * G.abs())).sum(-1)
            a, ra = self.a[s], self.ra[s]
            ah = a * self.hs[s]
            eah = a * self.ehs[s] + (ra + U) * ah.abs()
            t, et = G * ah, eG * ah.abs() + G.abs() * (eah + U * ah.abs())
            w[:, s], ew[:, s] = (t * self.A).sum(-1), (self.A.abs() * (et + terms * U * t.abs())).sum(-1)
            d, ed = self.d[:, s, :, None], self.ed[:, s, :, None]
            dA += (t * d).sum(0)
            eA += (et * d.abs() + t.abs() * (ed + steps * U * d.abs())).sum(0)
            eG = a * eG + (ra + 2 * U) * (a * G).abs()
            G = a * G
        dd = self.u * q + w
        edd = self.u.abs() * eq + ew + 2 * U * ((self.u * q).abs() + w.abs())
        if self.softplus:
            sg = torch.sigmoid(self.raw)
            edd = edd * sg + U * (10 + 4 * self.raw.abs().clamp(max=100.0)) * (dd * sg).abs()
            dd = dd * sg
        dd, edd = dd * live, edd * live
        du = self.d * q + self.D * dp
        edu = self.d.abs() * eq + self.ed * q.abs() + self.D.abs() * edp + 3 * U * ((self.d * q).abs() + (self.D * dp).abs())
        out.update(du=(du, edu), ddelta=(dd, edd), dB=(dB, eB), dC=(dC, eC))
        out = {k: (sweep(v * live, self.ns, self.reverse), sweep(e * live, self.ns, self.reverse)) for k, (v, e) in out.items()}
        out["dA"] = (dA, eA + TINY)
        out["dD"] = ((dp * self.u).sum((0, 1)), ((edp + steps * U * dp.abs()) * self.u.abs()).sum((0, 1)) + TINY)
        out["ddelta_bias"] = (dd.sum((0, 1)), (edd + steps * U * dd.abs()).sum((0, 1)) + TINY)
        out["dh0"] = (G, eG + TINY)
        return out


# ------------------------------------------------------------------- group norm

def group_norm(x, gamma, beta, G, act, eps):
    """y and its bound before rounding, mean, rstd [N][G], and what the backward needs.  Statistics are
    those of 64-bit sums, rounded; v = fma(x - mean, rstd gamma, beta'): a few U of its terms."""
    N, C = x.shape[0], x.shape[-1]
    xg = x.to(F64).reshape(N, -1, G, C // G)
    mean = xg.mean((1, 3), keepdim=True)
    var = ((xg - mean) ** 2).mean((1, 3), keepdim=True)
    rstd = (var + eps) ** -0.5
    # sums of squares in 64 bits
    extra = 2.0 ** -50 * (1 + mean ** 2 / (var + eps))
    xh = ((xg - mean) * rstd).reshape(x.shape)
    gamma, beta = gamma.to(F64), beta.to(F64)
    v = xh * gamma + beta
    rel = extra.expand_as(xg).reshape(x.shape)
    ev = (xh * gamma).abs() * (6 * U + rel) + 3 * U * beta.abs() + 2 * U * v.abs()
    y, _, ey, _ = act_of(v, ev, act)
    return (y, ey), (mean[:, 0, :, 0], rstd[:, 0, :, 0]), (xh, mean, rstd, v)


def group_norm_backward(kept, x, gamma, beta, dy, G, act):
    xh, mean, rstd, v = kept
    N, C = x.shape[0], x.shape[-1]
    shape = (N, -1, G, C // G)
    gamma, beta, dy = gamma.to(F64), beta.to(F64), dy.to(F64)
    # the backward's differences are those of the rounded mean, its rstd a rounded one
    exh = (U * mean.abs() * rstd + 4 * U * xh.reshape(shape).abs()).reshape(x.shape)
    ev = gamma.abs() * exh + 2 * U * ((gamma * xh).abs() + beta.abs())
    _, slope, _, es = act_of(v, ev, act)
    dv, edv = dy * slope, dy.abs() * (es + U * slope.abs())
    rows = x.numel() // C
    chain = (rows + 8) * U
    axes = tuple(range(x.dim() - 1))
    dgamma = (dv * xh).sum(axes)
    eg = (edv * xh.abs() + dv.abs() * (exh + chain * xh.abs())).sum(axes) + TINY
    dbeta, eb = dv.sum(axes), (edv + chain * dv.abs()).sum(axes) + TINY
    a, ea = (gamma * dv).reshape(shape), (gamma.abs() * edv).reshape(shape)
    xg, exg = xh.reshape(shape), exh.reshape(shape)
    m1, m2 = a.mean((1, 3), keepdim=True), (a * xg).mean((1, 3), keepdim=True)
    em1 = (ea + chain * a.abs()).mean((1, 3), keepdim=True)
    em2 = (ea * xg.abs() + a.abs() * (exg + chain * xg.abs())).mean((1, 3), keepdim=True)
    dx = rstd * (a - m1 - xg * m2)
    edx = rstd * (ea + em1 + xg.abs() * em2 + exg * m2.abs() + 4 * U * (a.abs() + m1.abs() + (xg * m2).abs())) + 2 * U * dx.abs()
    return (dx.reshape(x.shape), edx.reshape(x.shape)), (dgamma, eg), (dbeta, eb)


# ------------------------------------------------------------------------ AdamW

def mix32(x):
    x = (x ^ (x >> 16)) * 0x7feb352d & 0xffffffff
    x = (x ^ (x >> 15)) * 0x846ca68b & 0xffffffff
    return x ^ (x >> 16)


def code_value(k, exponents):
    """What a code stands for, as a share of its scale."""
    E = (1 << exponents) - 1
    return k / 8 * 2.0 ** (1 - E) if k < 8 else (1 + k % 8 / 8) * 2.0 ** (k // 8 - E)


def code_of(r, exponents, random):
    """The code of a ratio in [0, 1] by 16 random bits: the one at or below it, or the next, by the first 16
    binary digits of how far r is between them."""
    low = 1 - ((1 << exponents) - 1)
    e = low
    while e < 0 and 2.0 ** (e + 1) <= r:
        e += 1
    steps = r * 2.0 ** (3 - e)                  # exact
    k = int(steps)
    frac = int((steps - k) * 65536)
    return k + 8 * (e - low) + (1 if frac + random >= 65536 else 0)


def adamw(p, g, m, v, t, lr, betas, eps, decay, scale=1.0):
    """p with its bound, and the new moments as fp32 numbers: rounded once from 64 bits."""
    (b1, b2), g = betas, g.to(F64) * scale
    m = (m.to(F64) * b1 + g * (1 - b1)).float()
    v = (v.to(F64) * b2 + g * g * (1 - b2)).float()
    step = m.to(F64) / (1 - b1 ** t) / ((v.to(F64) / (1 - b2 ** t)).sqrt() + eps)
    new = p.to(F64) - lr * (step + decay * p.to(F64))
    bound = lr * U * (10 * step.abs() + 4 * decay * p.to(F64).abs()) + U * new.abs() + TINY
    return new, bound, m, v


def narrow(x, exponents, halves):
    """(codes, scales) of an fp32 tensor; halves: 16 random bits an element."""
    x = x.reshape(-1)
    codes, scales = [], []
    for first in range(0, x.numel(), 256):
        block = x[first:first + 256].tolist()
        top = max(abs(a) for a in block)
        finite = top < float("inf") and all(a == a for a in block)
        scales.append(top if finite else float("nan"))
        for j, a in enumerate(block):
            if not finite or top == 0:
                codes.append(0)
                continue
            k = code_of(abs(a) / top, exponents, halves[first + j])
            if exponents == 5:
                k = 1 if a > 0 and k == 0 else k
            elif k and a < 0:
                k |= 128
            codes.append(k)
    return torch.tensor(codes, dtype=torch.uint8), torch.tensor(scales, dtype=torch.float32)


def wide(codes, scales, exponents):
    """The fp32 numbers that codes stand for."""
    table = torch.tensor([code_value(k & 127 if exponents == 4 else k, exponents) * (-1 if exponents == 4 and k > 127 else 1)
                          for k in range(256)], dtype=F64)
    return (table[codes.long()] * scales.to(F64).repeat_interleave(256)[:codes.numel()]).float()


def halves_of(n, seed, t, k, first=0):
    """The low and high 16 random bits of n elements of tensor k from element `first` on."""
    key = mix32((mix32((mix32(seed & 0xffffffff) + t) & 0xffffffff) + k) & 0xffffffff)
    r = [mix32((i & 0xffffffff) ^ key ^ mix32(i >> 32)) for i in range(first, first + n)]
    return [a & 0xffff for a in r], [a >> 16 for a in r]


__all__ = ["rounded"]
