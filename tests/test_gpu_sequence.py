"""Layer norm, the gated linear scan and 8-bit checkpoints on the GPU, against
the plain 64-bit forms of tests/seq_ref.py with their bounds."""
from __future__ import annotations

import pytest
import torch

import paper_1506_07452_amd as P
from tests import seq_ref as R
from tests.gpu_util import DEV, say

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
IDS = {F32: "f32", BF16: "bf16"}
DTYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
FILL = 77.0


def rand(seed, shape, dtype, scale=1.0, shift=0.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * scale + shift).to(dtype)


class Out:
    """A device output between guard bands that a kernel must leave alone."""

    def __init__(self, shape, dtype):
        n = 1
        for e in shape:
            n *= e
        fill = 77 if dtype == torch.int8 else FILL
        self.whole = torch.full((n + 512,), fill, dtype=dtype, device=DEV)
        self.n, self.fill = n, fill
        self.t = self.whole[256:256 + n].view(shape)

    def get(self):
        assert (self.whole[:256] == self.fill).all() and (self.whole[256 + self.n:] == self.fill).all(), \
            "written outside the output"
        return self.t.cpu()


def near(name, got, value, bound):
    got = got.double()
    assert got.shape == value.shape, name
    off = (got - value).abs()
    worst = (off / bound).max()
    assert torch.isfinite(got).all(), name + " is not finite"
    assert bool((off <= bound).all()), "%s off by %.3g of its bound (%.3g)" % (
        name, float(worst), float(off.max()))


# ------------------------------------------------------------------ layer norm

def norm_step(M, C, dtype, ckpt=False, want_dx=True, seed=0, x=None, stream=None):
    x = rand(seed, (M, C), dtype, 0.8, 0.3) if x is None else x
    gamma, beta = rand(seed + 1, (C,), dtype, 0.2, 1.0), rand(seed + 2, (C,), dtype, 0.1)
    dy = rand(seed + 3, (M, C), dtype, 0.1)
    dx_, dev = None, [t.to(DEV) for t in (x, gamma, beta, dy)]
    y, stats = Out((M, C), dtype), Out((M, 2), F32)
    dgamma, dbeta = Out((C,), F32), Out((C,), F32)
    q = Out((M, C), torch.int8) if ckpt else None
    qs = Out((-(-M * C // 64),), BF16) if ckpt else None
    P.pyramid_layer_norm_forward(dev[0], dev[1], dev[2], y.t, stats.t, q.t if ckpt else None,
                                 qs.t if ckpt else None, stream=stream)
    if want_dx:
        dx_ = Out((M, C), dtype)
    P.pyramid_layer_norm_backward(q.t if ckpt else dev[0], dev[1], stats.t, dev[3],
                                  dx_.t if want_dx else None, dgamma.t, dbeta.t,
                                  xscale=qs.t if ckpt else None, stream=stream)
    torch.cuda.synchronize()
    ry, by, mean, rstd = R.norm_forward(x, gamma, beta, 1e-5, dtype)
    near("y", y.get(), ry, by)
    kept = x
    if ckpt:
        rq, rs, kept = R.codes(x)
        assert torch.equal(q.get(), rq) and torch.equal(qs.get(), rs)
    dx, dg, db = R.norm_backward(kept, mean, rstd, gamma, dy, dtype)
    near("mean", stats.get()[:, 0], mean[:, 0], 64 * R.U * x.double().abs().amax(1) + R.TINY)
    near("rstd", stats.get()[:, 1], rstd[:, 0],
         rstd[:, 0] * R.U * (40 + 70 * x.double().abs().amax(1) * rstd[:, 0]))
    if want_dx:
        near("dx", dx_.get(), *dx)
    near("dgamma", dgamma.get(), *dg)
    near("dbeta", dbeta.get(), *db)


@DTYPES
@pytest.mark.parametrize("C", [1, 2, 3, 4, 7, 8, 15, 16, 17, 25, 32, 45, 63, 64, 65, 90, 128, 129, 255, 256, 257,
                               500, 512, 513, 1000, 1023, 1024, 1025])
def test_norm_channels(C, dtype):
    say("norm", C, dtype)
    norm_step(37, C, dtype)


@DTYPES
@pytest.mark.parametrize("C", [2000, 2048, 2049, 4096, 4099, 8192, 8193, 12288, 16383, 16384])
def test_norm_wide(C, dtype):
    say("norm wide", C, dtype)
    norm_step(5, C, dtype)


@DTYPES
@pytest.mark.parametrize("M", [1, 2, 3, 15, 16, 17, 63, 64, 65, 255, 257, 1000, 4099])
@pytest.mark.parametrize("C", [16, 45])
def test_norm_rows(M, C, dtype):
    say("norm rows", M, C, dtype)
    norm_step(M, C, dtype, seed=M)


@DTYPES
@pytest.mark.parametrize("M,C", [(1, 1), (7, 1), (65, 3), (33, 8), (9, 16), (130, 16), (50, 32), (77, 64), (20, 45),
                                 (31, 128), (12, 192), (9, 320), (6, 1024), (3, 2048), (3, 5000), (2, 8192), (2, 16384),
                                 (300, 45), (64, 45), (65, 25), (1000, 5), (513, 7), (129, 12), (200, 63), (100, 33),
                                 (70, 90), (65, 100), (33, 130), (40, 250), (30, 131), (600, 2), (257, 17), (90, 500)])
def test_norm_from_checkpoint(M, C, dtype):
    say("norm ckpt", M, C, dtype)
    norm_step(M, C, dtype, ckpt=True, seed=M + C)


@DTYPES
@pytest.mark.parametrize("C", [16, 45, 2048, 9000])
def test_norm_without_dx(C, dtype):
    say("norm no dx", C, dtype)
    norm_step(70, C, dtype, want_dx=False)


@DTYPES
def test_norm_far_from_zero(dtype):
    """Rows whose mean is far above their spread: the variance is that of the
    differences, not of the squares."""
    x = rand(5, (40, 96), F32, 1.0, 200.0).to(dtype)
    say("norm far", dtype)
    norm_step(40, 96, dtype, x=x)


def test_norm_constant_rows_and_infinities():
    """A constant row has xh = 0; a row with an infinity or a NaN is NaN, its
    neighbours are not touched."""
    M, C = 70, 48
    x = rand(3, (M, C), F32)
    x[4] = 2.5
    x[7, 3], x[9, 47] = float("inf"), float("nan")
    gamma, beta = rand(1, (C,), F32, 0.2, 1.0), rand(2, (C,), F32)
    y, stats = Out((M, C), F32), Out((M, 2), F32)
    say("norm special rows")
    P.pyramid_layer_norm_forward(x.to(DEV), gamma.to(DEV), beta.to(DEV), y.t, stats.t)
    got = y.get()
    assert torch.equal(got[4], beta)
    assert torch.isnan(got[7]).all() and torch.isnan(got[9]).all()
    rest = [m for m in range(M) if m not in (7, 9)]
    ry, by, _, _ = R.norm_forward(x[rest], gamma, beta, 1e-5, F32)
    near("y", got[rest], ry, by)


def test_norm_is_repeatable_and_follows_differences():
    """The same call twice gives the same bits; dx follows differences of the
    64-bit form's loss."""
    M, C = 300, 45
    x, dy = rand(1, (M, C), F32), rand(2, (M, C), F32)
    gamma, beta = rand(3, (C,), F32, 0.2, 1.0), rand(4, (C,), F32)
    dev = [t.to(DEV) for t in (x, gamma, beta, dy)]
    out = []
    for _ in range(2):
        y, stats = torch.empty_like(dev[0]), torch.empty((M, 2), device=DEV)
        dx, dg, db = torch.empty_like(y), torch.empty(C, device=DEV), torch.empty(C, device=DEV)
        P.pyramid_layer_norm_forward(dev[0], dev[1], dev[2], y, stats)
        P.pyramid_layer_norm_backward(dev[0], dev[1], stats, dev[3], dx, dg, db)
        out.append([t.cpu() for t in (y, stats, dx, dg, db)])
    assert all(torch.equal(a, b) for a, b in zip(*out))
    # directional differences: f(x + h v) - f(x - h v) over 2 h, error h^2 f'''/6
    step, dirs = 1e-4, [rand(10 + k, (M, C), F32).double() for k in range(3)]
    for v in dirs:
        f = [float((R.norm_forward(x.double() + k * step * v, gamma, beta, 1e-5, F32)[0] * dy.double()).sum())
             for k in (1, -1)]
        want = (f[0] - f[1]) / (2 * step)
        got = float((out[0][2].double() * v).sum())
        assert abs(got - want) <= 1e-5 * float((out[0][2].double() * v).abs().sum())


def test_norm_past_32_bit_offsets():
    """2^31 + elements: rows at the end are right, in both passes."""
    C, M = 1024, (1 << 21) + 5
    x = torch.empty((M, C), dtype=BF16, device=DEV)
    x.normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    gamma, beta = rand(1, (C,), BF16, 0.2, 1.0), rand(2, (C,), BF16)
    y, stats = torch.zeros_like(x), torch.zeros((M, 2), device=DEV)
    dg, db = torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    say("norm past 2^31")
    P.pyramid_layer_norm_forward(x, gamma.to(DEV), beta.to(DEV), y, stats)
    dx = torch.zeros_like(x)
    P.pyramid_layer_norm_backward(x, gamma.to(DEV), stats, x, dx, dg, db)
    for at in (0, M - 6):
        rows = x[at:at + 6].cpu()
        ry, by, mean, rstd = R.norm_forward(rows, gamma, beta, 1e-5, BF16)
        near("y", y[at:at + 6].cpu(), ry, by)
        near("dx", dx[at:at + 6].cpu(), *R.norm_backward(rows, mean, rstd, gamma, rows, BF16)[0])
    near("dbeta", db.cpu(), x.sum(0, dtype=torch.float64).cpu(),
         (64 + M / 256) * R.U * x.abs().sum(0, dtype=torch.float64).cpu())


# ------------------------------------------------------------------------ scan

def scan_step(B, T, I, dtype, reverse=False, lengths=None, state=True, ckpt=False, seed=0, g=None, u=None,
              poison=True, shift=1.0):
    g = rand(seed, (B, T, I), dtype, 1.5, shift) if g is None else g
    u = rand(seed + 1, (B, T, I), dtype) if u is None else u
    dh = rand(seed + 2, (B, T, I), dtype, 0.3)
    h0 = rand(seed + 3, (B, I), F32) if state else None
    dhT = rand(seed + 4, (B, I), F32) if state else None
    if lengths is not None and poison and not ckpt:
        for b, n in enumerate(lengths):     # what a sequence does not have is not read
            for v in (g, u, dh):
                v[b, min(max(n, 0), T):] = float("nan")
    dev = lambda t: None if t is None else t.to(DEV)    # noqa: E731
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).to(DEV)
    dg_, du_, h_ = Out((B, T, I), dtype), Out((B, T, I), dtype), Out((B, T, I), dtype)
    hT_, dh0_ = Out((B, I), F32), Out((B, I), F32)
    nbytes = P.pyramid_scan_saved_size(B, T, I)
    saved = Out((nbytes // 4,), F32)
    gd, ud = dev(g), dev(u)
    P.pyramid_scan_forward(gd, ud, h_.t, reverse, ln, dev(h0), hT_.t if state else None, saved.t)
    gs = us = None
    gk, uk, gr, ur = gd, ud, g, u
    if ckpt:
        gk, gs = P.checkpoint8_empty(gd)
        uk, us = P.checkpoint8_empty(ud)
        P.pyramid_checkpoint8_pack(gd, gk, gs)
        P.pyramid_checkpoint8_pack(ud, uk, us)
        gr, ur = R.codes(g)[2], R.codes(u)[2]
    P.pyramid_scan_backward(gk, uk, saved.t, dev(dh), dg_.t, du_.t, reverse, ln, dev(dhT),
                            dh0_.t if state else None, gscale=gs, uscale=us)
    torch.cuda.synchronize()
    h, e, hT, eT, before, eb = R.scan_forward(g, u, reverse, lengths, h0)
    near("h", h_.get(), h, R.rounded(h, e, dtype))
    if state:
        near("hT", hT_.get(), hT, eT)
    saved.get()
    if ckpt:
        before, eb = R.scan_forward(gr, ur, reverse, lengths, h0, run=(before, eb))[4:]
    (dg, eg), (du, eu), (dh0, e0) = R.scan_backward(gr, ur, before, eb, dh, reverse, lengths, dhT)
    near("dg", dg_.get(), dg, R.rounded(dg, eg, dtype))
    near("du", du_.get(), du, R.rounded(du, eu, dtype))
    if state:
        near("dh0", dh0_.get(), dh0, e0)


@DTYPES
@pytest.mark.parametrize("reverse", [False, True], ids=["fwd", "rev"])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 127, 128, 130, 255, 256, 257, 300, 511, 513, 1030])
def test_scan_lengths(T, reverse, dtype):
    say("scan T", T, reverse, dtype)
    scan_step(2, T, 24, dtype, reverse, seed=T)


@DTYPES
@pytest.mark.parametrize("I", [1, 2, 3, 4, 5, 7, 8, 12, 16, 31, 32, 63, 64, 65, 100, 127, 128, 130, 192, 256, 260, 333, 513])
def test_scan_channels(I, dtype):
    say("scan I", I, dtype)
    scan_step(3, 50, I, dtype, reverse=I % 2 == 1, seed=I)


@DTYPES
@pytest.mark.parametrize("I", [1, 6, 64, 130])
def test_scan_long(I, dtype):
    say("scan long", I, dtype)
    scan_step(1, 5003, I, dtype, reverse=I == 64, seed=I, shift=3.0)


@DTYPES
@pytest.mark.parametrize("B,T,I", [(40, 20, 16), (257, 9, 4), (1000, 5, 3), (65, 33, 1), (300, 40, 16)])
def test_scan_many_sequences(B, T, I, dtype):
    say("scan B", B, T, I, dtype)
    scan_step(B, T, I, dtype, reverse=True, seed=B)


RAGGED = [([0, 1, 40, 7, 16, 39, 17], 40, 5), ([0], 3, 2), ([3, 0, 0], 3, 70), ([600, 0, 599, 256, 257, 1], 600, 36),
          ([-4, 900, 33], 50, 64), ([1500, 17], 1500, 128)]


@DTYPES
@pytest.mark.parametrize("reverse", [False, True], ids=["fwd", "rev"])
@pytest.mark.parametrize("lengths,T,I", RAGGED)
def test_scan_ragged(lengths, T, I, reverse, dtype):
    say("scan ragged", lengths, T, I, reverse, dtype)
    scan_step(len(lengths), T, I, dtype, reverse, lengths, seed=T)


@DTYPES
def test_scan_ragged_many_short_sequences(dtype):
    n = [(7 * k) % 24 for k in range(200)]
    say("scan ragged many", dtype)
    scan_step(200, 23, 4, dtype, True, n, seed=9)


@DTYPES
@pytest.mark.parametrize("state", [False, True], ids=["zero", "state"])
@pytest.mark.parametrize("B,T,I", [(1, 1, 1), (2, 40, 16), (3, 33, 7), (1, 700, 64), (2, 300, 130), (90, 37, 16)])
def test_scan_from_checkpoint(B, T, I, state, dtype):
    say("scan ckpt", B, T, I, dtype)
    scan_step(B, T, I, dtype, reverse=T % 2 == 1, state=state, ckpt=True, seed=B + T)


@DTYPES
def test_scan_ragged_from_checkpoint(dtype):
    say("scan ragged ckpt", dtype)
    scan_step(4, 290, 33, dtype, True, [0, 290, 17, 288], ckpt=True, seed=4)


def test_scan_gates_at_the_ends():
    """Gates of +-infinity and of the type's largest and lowest values: f is
    0 or 1, the state is replaced or kept, gradients of g are 0."""
    for dtype in (F32, BF16):
        g = rand(1, (2, 90, 8), dtype, 3.0)
        big = torch.finfo(dtype).max
        g[0, 3], g[0, 20], g[1, 50], g[1, 7] = float("inf"), -float("inf"), big, -big
        g[0, 40:60], g[1, 60:] = -float("inf"), float("inf")
        say("scan ends", dtype)
        scan_step(2, 90, 8, dtype, g=g, seed=1)
        scan_step(2, 90, 8, dtype, reverse=True, g=g, seed=1)


def test_scan_nan_goes_forward_from_its_step():
    g, u = rand(1, (2, 600, 70), F32), rand(2, (2, 600, 70), F32)
    u[1, 300, 5] = float("nan")
    h = Out((2, 600, 70), F32)
    say("scan nan")
    P.pyramid_scan_forward(g.to(DEV), u.to(DEV), h.t)
    got = h.get()
    assert torch.isnan(got[1, 300:, 5]).all()
    got[1, 300:, 5] = 0
    ref, e = R.scan_forward(g, u.nan_to_num(0.0), False, None, None)[:2]
    ref[1, 300:, 5] = 0
    near("h", got, ref, R.rounded(ref, e, F32))


@DTYPES
def test_scan_long_memory(dtype):
    """Gates that keep all but 1e-6 to 1e-3 of the state, 4000 steps."""
    say("scan memory", dtype)
    scan_step(1, 4000, 20, dtype, g=rand(1, (1, 4000, 20), dtype, 1.0, 10.0), seed=1)


@DTYPES
@pytest.mark.parametrize("B,I", [(1, 1), (16, 2048), (3, 333)])
def test_scan_single_steps_carry_the_state_in_place(B, I, dtype):
    """T = 1 calls with hT = h0 give what one call over all steps gives; so
    does a sequence cut into chunks of other lengths."""
    T = 37
    g, u, start = rand(1, (B, T, I), dtype, 1.5, 1.0), rand(2, (B, T, I), dtype), rand(3, (B, I), F32)
    h, e, hT, eT = R.scan_forward(g, u, False, None, start)[:4]
    gd, ud = g.to(DEV), u.to(DEV)
    say("scan steps", B, I, dtype)
    for cuts in ([1] * T, [5, 16, 1, 15], [T]):
        st, t = Out((B, I), F32), 0
        st.t.copy_(start)
        for n in cuts:
            part = Out((B, n, I), dtype)
            P.pyramid_scan_forward(gd[:, t:t + n].contiguous(), ud[:, t:t + n].contiguous(), part.t, h0=st.t, hT=st.t)
            near("h", part.get(), h[:, t:t + n], R.rounded(h, e, dtype)[:, t:t + n])
            t += n
        near("hT", st.get(), hT, eT)


def test_scan_gradient_follows_differences():
    B, T, I = 2, 300, 6
    g, u, dh = (rand(k, (B, T, I), F32) for k in (1, 2, 3))
    h0 = rand(4, (B, I), F32)
    dev = [t.to(DEV) for t in (g, u, dh, h0)]
    saved = torch.empty(P.pyramid_scan_saved_size(B, T, I), dtype=torch.uint8, device=DEV)
    h, dg, du, dh0 = torch.empty_like(dev[0]), torch.empty_like(dev[0]), torch.empty_like(dev[0]), torch.empty_like(dev[3])
    P.pyramid_scan_forward(dev[0], dev[1], h, True, h0=dev[3], saved=saved)
    P.pyramid_scan_backward(dev[0], dev[1], saved, dev[2], dg, du, True, dh0=dh0)
    step = 1e-4     # the difference's own error: step^2 / 6 of the third derivative, below 1e-7
    for k, grad in enumerate((dg, du, dh0)):
        v = rand(20 + k, grad.shape, F32).double()
        f = []
        for sgn in (1, -1):
            a = [g.double(), u.double(), h0.double()]
            a[k] = a[k] + sgn * step * v
            f.append(float((R.scan_forward(a[0], a[1], True, None, a[2])[0] * dh.double()).sum()))
        got = float((grad.cpu().double() * v).sum())
        assert abs(got - (f[0] - f[1]) / (2 * step)) <= 1e-5 * float((grad.cpu().double() * v).abs().sum())


def test_scan_is_repeatable():
    B, T, I = 1, 9000, 128
    g, u, dh = (rand(k, (B, T, I), F32).to(DEV) for k in (1, 2, 3))
    saved = torch.empty(P.pyramid_scan_saved_size(B, T, I), dtype=torch.uint8, device=DEV)
    first = None
    say("scan repeat")
    for _ in range(4):
        h, dg, du = (torch.empty_like(g) for _ in range(3))
        P.pyramid_scan_forward(g, u, h, saved=saved)
        P.pyramid_scan_backward(g, u, saved, dh, dg, du)
        now = [h, dg, du]
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


@pytest.mark.parametrize("B,T,I", [((1 << 11) + 3, 64, 16384), (1, (1 << 20) + 33, 2049)], ids=["columns", "steps"])
def test_scan_past_32_bit_offsets(B, T, I):
    """More than 2^31 elements: the last columns and steps, forward and backward."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    g, u = (torch.empty((B, T, I), dtype=BF16, device=DEV).normal_(generator=gen) for _ in range(2))
    h, dg, du = torch.empty_like(g), torch.empty_like(g), torch.empty_like(g)
    saved = torch.empty(P.pyramid_scan_saved_size(B, T, I), dtype=torch.uint8, device=DEV)
    say("scan past 2^31", B, T, I)
    P.pyramid_scan_forward(g, u, h, saved=saved)
    P.pyramid_scan_backward(g, u, saved, u, dg, du)
    cols = [0, I - 1]
    # gates of mean 1/2 forget within 64 steps: 2^-64 of the state before is below every bound
    t0 = max(0, T - 200)
    gl, ul = (v[-1:, t0:][:, :, cols].cpu() for v in (g, u))
    rh, e, _, _, before, eb = R.scan_forward(gl, ul, False, None, None)
    near("h", h[-1:, t0 + 100 if t0 else 0:][:, :, cols].cpu(), *[v[:, 100 if t0 else 0:] for v in (rh, R.rounded(rh, e, BF16))])
    (rg, eg), (ru, eu), _ = R.scan_backward(gl, ul, before, eb, ul, False, None, None)
    k = 100 if t0 else 0
    near("dg", dg[-1:, t0 + k:][:, :, cols].cpu(), rg[:, k:], R.rounded(rg, eg, BF16)[:, k:])
    near("du", du[-1:, t0 + k:][:, :, cols].cpu(), ru[:, k:], R.rounded(ru, eu, BF16)[:, k:])


# ------------------------------------------------------------------ checkpoints

def ckpt_step(x):
    q, s, back = Out(x.shape, torch.int8), Out((-(-x.numel() // 64),), BF16), Out(x.shape, x.dtype)
    P.pyramid_checkpoint8_pack(x.to(DEV), q.t, s.t)
    P.pyramid_checkpoint8_unpack(q.t, s.t, back.t)
    torch.cuda.synchronize()
    rq, rs, rv = R.codes(x)
    for name, got, want in (("scale", s.get(), rs), ("codes", q.get(), rq), ("values", back.get(), rv.to(x.dtype))):
        same = (got == want) | ((got != got) & (want != want))      # a NaN is a NaN whatever its bits
        assert bool(same.all()), (name, int((~same).sum()), got[~same][:4], want[~same][:4])


@DTYPES
@pytest.mark.parametrize("n", [1, 2, 3, 15, 16, 17, 63, 64, 65, 100, 127, 128, 129, 255, 256, 1000, 1023, 1024, 1025,
                               4095, 4097, 12345, 65536, 1000003])
def test_checkpoint_sizes(n, dtype):
    say("ckpt", n, dtype)
    x = rand(n, (n,), F32) * torch.exp2(torch.floor(rand(n + 1, (n,), F32, 2.0)))
    ckpt_step(x.to(dtype))


@DTYPES
def test_checkpoint_ties_and_their_neighbours(dtype):
    """Values on and one step beside every half code, at scales of every
    mantissa: the nearest code, ties to the even one."""
    blocks = []
    for m in range(128, 256):
        s = m * 2.0 ** (m % 40 - 20)
        ties = torch.tensor([(k + 0.5) * s for k in range(-127, 127)], dtype=torch.float64).to(dtype)
        if dtype == F32:
            vals = torch.cat([ties, torch.nextafter(ties, torch.tensor(1e30)), torch.nextafter(ties, torch.tensor(-1e30))])
        else:
            vals = ties
        vals = vals[: vals.numel() // 63 * 63].view(-1, 63)
        top = torch.full((vals.shape[0], 1), 127.0 * s, dtype=torch.float64).to(dtype)
        blocks.append(torch.cat([top, vals], 1))
    say("ckpt ties", dtype)
    ckpt_step(torch.cat(blocks))


@DTYPES
def test_checkpoint_magnitudes(dtype):
    """Blocks from the smallest denormals to the largest numbers, zeros, and
    blocks with infinities and NaN beside ordinary ones."""
    rows = [rand(e, (64,), F32).clamp(-3, 3).double() * 2.0 ** e for e in range(-150, 126, 3)]
    x = torch.stack(rows).to(dtype)
    x[5] = 0
    x[7, 11], x[9, 0], x[11, 63], x[13, 13] = float("inf"), float("nan"), -float("inf"), torch.finfo(dtype).max
    x[14] = -0.0
    for k, e in enumerate((-120, -119, -118)):      # around the smallest scale
        x[20 + k] = torch.full((64,), 2.0 ** e).to(dtype)
        x[20 + k, 5] = (x[20 + k, 5].double() * 0.995).to(dtype)
    say("ckpt magnitudes", dtype)
    ckpt_step(x)


def test_checkpoint_past_32_bit_offsets():
    n = (1 << 31) + 12345
    x = torch.zeros(n, dtype=BF16, device=DEV)
    tail = rand(1, (5000,), BF16)
    x[-5000:] = tail.to(DEV)
    q, s = P.checkpoint8_empty(x)
    say("ckpt past 2^31")
    P.pyramid_checkpoint8_pack(x, q, s)
    back = torch.empty_like(x)
    P.pyramid_checkpoint8_unpack(q, s, back)
    at = n - n % 64 - 64 * 64
    assert torch.equal(back[at:].cpu(), R.codes(x[at:].cpu())[2].to(BF16))
    assert not back[:1 << 20].any()


# --------------------------------------------------- streams, graphs, refusals

def block_step(x, w, reverse, ckpt):
    """Norm, then a scan of the normed rows as inputs with themselves as gates,
    and back: what a pre-normed recurrent block does."""
    B, T, I = x.shape
    y, stats = torch.empty_like(x), torch.empty((B * T, 2), device=DEV)
    rows = x.view(B * T, I)
    kept, ks = P.checkpoint8_empty(rows) if ckpt else (rows, None)
    P.pyramid_layer_norm_forward(rows, w[0], w[1], y.view(B * T, I), stats, kept if ckpt else None, ks)
    h = torch.empty_like(x)
    saved = torch.empty(P.pyramid_scan_saved_size(B, T, I), dtype=torch.uint8, device=DEV)
    P.pyramid_scan_forward(x, y, h, reverse, saved=saved)
    gk, gs, uk, us = x, None, y, None
    if ckpt:
        gk, gs = kept.view(B, T, I), ks
        uk, us = P.checkpoint8_empty(y)
        P.pyramid_checkpoint8_pack(y, uk, us)
    dg, du = torch.empty_like(x), torch.empty_like(x)
    P.pyramid_scan_backward(gk, uk, saved, h, dg, du, reverse, gscale=gs, uscale=us)
    dx = torch.empty_like(rows)
    dgamma, dbeta = torch.empty(I, device=DEV), torch.empty(I, device=DEV)
    P.pyramid_layer_norm_backward(kept, w[0], stats, du.view(B * T, I), dx, dgamma, dbeta, xscale=ks)
    return [h, dg, du, dx, dgamma, dbeta]


@DTYPES
@pytest.mark.parametrize("B,T,I,ckpt", [(2, 40, 48, False), (1, 3000, 64, True), (4, 700, 33, True), (1, 5000, 256, False)])
def test_operators_in_a_graph_and_on_streams(B, T, I, ckpt, dtype):
    """A captured step replayed with eager work and other inputs between the
    replays, a second graph beside it, and two streams at once, against eager
    results."""
    x = rand(1, (B, T, I), dtype, 1.0, 0.5).to(DEV)
    other = rand(2, (B, T, I), dtype).to(DEV)
    w = [rand(3, (I,), dtype, 0.2, 1.0).to(DEV), rand(4, (I,), dtype).to(DEV)]
    say("graph", B, T, I, dtype)
    want = [t.clone() for t in block_step(x, w, False, ckpt)]
    want_other = [t.clone() for t in block_step(other, w, True, ckpt)]
    torch.cuda.synchronize()
    static = [x.clone(), other.clone()]
    graphs, outs = [], []
    for k in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(block_step(static[k], w, k == 1, ckpt))
        graphs.append(graph)
    for turn in range(3):
        static[0].copy_(x)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[0], want)), turn
        assert all(torch.equal(a, b) for a, b in zip(outs[1], want_other)), turn
        # other inputs through the same graph, eager work beside it
        static[0].copy_(other)
        graphs[0].replay()
        eager = block_step(other, w, False, ckpt)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[0], eager)), turn
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for k, st in enumerate(streams):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            got.append(block_step(x if k == 0 else other, w, k == 1, ckpt))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got[0], want))
    assert all(torch.equal(a, b) for a, b in zip(got[1], want_other))


@pytest.mark.parametrize("raw", [False, True], ids=["stream", "handle"])
def test_workspace_belongs_to_the_calls_stream(raw):
    """A call given another stream than the current one, which is still busy
    when the call returns: its workspace is not handed to the next tensors of
    the current stream."""
    M, C = 4096, 1024
    x, dy = rand(1, (M, C), F32).to(DEV), rand(2, (M, C), F32).to(DEV)
    w = [rand(3, (C,), F32, 0.2, 1.0).to(DEV), rand(4, (C,), F32).to(DEV)]
    g, u = rand(5, (1, 6000, 256), F32).to(DEV), rand(6, (1, 6000, 256), F32).to(DEV)
    a = torch.randn(4096, 4096, device=DEV)

    def calls(stream):
        y, stats, dx = torch.empty_like(x), torch.empty((M, 2), device=DEV), torch.empty_like(x)
        dg, db, h = torch.empty(C, device=DEV), torch.empty(C, device=DEV), torch.empty_like(g)
        if stream is not None:
            torch.cuda.synchronize()        # the outputs' memory is free
            with torch.cuda.stream(stream):
                for _ in range(20):
                    a @ a
            if raw:
                stream = stream.cuda_stream
        P.pyramid_layer_norm_forward(x, w[0], w[1], y, stats, stream=stream)
        P.pyramid_layer_norm_backward(x, w[0], stats, dy, dx, dg, db, stream=stream)
        P.pyramid_scan_forward(g, u, h, stream=stream)
        return [y, dx, dg, db, h]

    want = calls(None)
    side = torch.cuda.Stream()
    say("workspace and stream", raw)
    got = calls(side)
    junk = [torch.full((P.pyramid_layer_norm_workspace_size(M, C) // 4,), float("nan"), device=DEV),
            torch.full((P.pyramid_scan_workspace_size(1, 6000, 256) // 4,), float("nan"), device=DEV)]
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    del junk


def test_refusals_of_the_binding():
    """Wrong shapes, types, places and layouts are refused before a launch."""
    x, v = torch.zeros((4, 8), device=DEV), torch.zeros(8, device=DEV)
    y = torch.zeros_like(x)
    for bad in (dict(gamma=torch.zeros(7, device=DEV)), dict(gamma=v.to(BF16)), dict(y=torch.zeros((8, 4), device=DEV)),
                dict(x=x.half()), dict(x=torch.zeros((8, 4), device=DEV).t()), dict(beta=torch.zeros(8)),
                dict(stats=torch.zeros((4, 3), device=DEV)), dict(xq=torch.zeros((4, 8), dtype=torch.int8, device=DEV))):
        a = dict(x=x, gamma=v, beta=v, y=y)
        a.update(bad)
        with pytest.raises(ValueError):
            P.pyramid_layer_norm_forward(**a)
    g = torch.zeros((2, 5, 8), device=DEV)
    for bad in (dict(u=g[:, :4].contiguous()), dict(h=g.to(BF16)), dict(lengths=torch.zeros(2, device=DEV)),
                dict(h0=torch.zeros((2, 8), dtype=BF16, device=DEV)), dict(saved=torch.zeros(4, device=DEV)),
                dict(g=g.transpose(0, 1)), dict(hT=torch.zeros((2, 7), device=DEV))):
        a = dict(g=g, u=g, h=torch.zeros_like(g))
        a.update(bad)
        with pytest.raises(ValueError):
            P.pyramid_scan_forward(**a)
    with pytest.raises(P.PyramidLSTMError):
        P.pyramid_layer_norm_forward(x[:0], v, v, y[:0])
    with pytest.raises(P.PyramidLSTMError):
        P.pyramid_scan_forward(g[:, :0], g[:, :0], g[:, :0].clone())
    with pytest.raises(ValueError):
        P.pyramid_checkpoint8_pack(x, torch.zeros((4, 8), dtype=torch.int8, device=DEV),
                                   torch.zeros(2, dtype=BF16, device=DEV))


@pytest.mark.parametrize("I", [517, 514])
def test_scan_sequences_far_apart(I):
    """Sequences too long for 32-bit offsets between them, whose columns would
    share a wave: the last steps of each."""
    B, T = 3, (1 << 20) + 33
    gen = torch.Generator(device=DEV).manual_seed(5)
    g, u = (torch.empty((B, T, I), dtype=BF16, device=DEV).normal_(generator=gen) for _ in range(2))
    lengths = [T, T - 5000, T - 77]
    ln = torch.tensor(lengths, dtype=torch.int32).to(DEV)
    say("scan far apart")
    for reverse in (False, True):
        for n in (None, ln):
            h, dg, du = (torch.full_like(g, FILL) for _ in range(3))
            saved = torch.empty(P.pyramid_scan_saved_size(B, T, I), dtype=torch.uint8, device=DEV)
            P.pyramid_scan_forward(g, u, h, reverse, n, saved=saved)
            P.pyramid_scan_backward(g, u, saved, u, dg, du, reverse, n)
            cols = [0, 1, I - 1]
            for b in range(B):
                end = T if n is None else lengths[b]
                # the sweep's last 200 positions; 100 steps before them are forgotten to 2^-64
                at = slice(0, 200) if reverse else slice(end - 200, end)
                gl, ul = (v[b:b + 1, at][:, :, cols].cpu() for v in (g, u))
                rh, e, _, _, before, eb = R.scan_forward(gl, ul, reverse, None, None)
                (rg, eg), (ru, eu), _ = R.scan_backward(gl, ul, before, eb, ul, reverse, None, None)
                keep = slice(0, 100) if reverse else slice(100, 200)
                for name, got, ref, err in (("h", h, rh, e), ("dg", dg, rg, eg), ("du", du, ru, eu)):
                    near(name, got[b:b + 1, at][:, :, cols].cpu()[:, keep], ref[:, keep],
                         R.rounded(ref, err, BF16)[:, keep])
                if end < T:
                    assert not h[b, end:].any() and not dg[b, end:].any() and not du[b, end:].any()


def test_scan_columns_past_a_wide_launch():
    """The most columns that there may be, of more than one run: 2^24 workgroups, which
    a launch takes with one wave each alone.  The columns repeat those of the first 341
    sequences (37 GB a tensor)."""
    P0, T, I = 341, 17, 63
    B = (1 << 30) // I
    assert B % P0 == 0 and B * I > (1 << 30) - 64
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 140 << 30:
        pytest.skip("needs 140 GB of free memory")
    one = rand(1, (P0, T, I), BF16, 1.5, 1.0)
    g = torch.empty((B, T, I), dtype=BF16, device=DEV)
    g.view(-1, P0, T, I).copy_(one.to(DEV))
    h, saved = torch.empty_like(g), torch.empty(P.pyramid_scan_saved_size(B, T, I), dtype=torch.uint8, device=DEV)
    say("scan of 2^30 columns")
    P.pyramid_scan_forward(g, g, h, True, saved=saved)

    def whole(name, t, ref, err):
        rows = t.view(B // P0, -1)
        near(name, t[:P0].cpu(), ref, R.rounded(ref, err, BF16))
        for k in range(0, rows.shape[0], 4096):
            assert bool((rows[k:k + 4096] == rows[:1]).all()), (name, k)

    ref, e, _, _, before, eb = R.scan_forward(one, one, True, None, None)
    whole("h", h, ref, e)
    dg, du = h, torch.empty_like(g)
    P.pyramid_scan_backward(g, g, saved, g, dg, du, True)
    (rg, eg), (ru, eu), _ = R.scan_backward(one, one, before, eb, one, True, None, None)
    whole("dg", dg, rg, eg)
    whole("du", du, ru, eu)
    del g, h, saved, dg, du
    torch.cuda.empty_cache()


def full_mantissa(seed, n):
    """fp32 values whose 24 bits are all in use, of magnitudes 1e-3 to 1e6, and three round ones in decimal."""
    v = rand(seed, (n,), F32) * 10.0 ** rand(seed + 1, (n,), F32, 2.0).clamp(-3, 6)
    v[:3] = torch.tensor([0.1, 1000.1, -33333.3])
    return v


@pytest.mark.parametrize("C", [2, 3, 7, 25, 45, 48, 64, 100, 130, 1000, 2048, 4096, 5000, 12001, 16384])
def test_norm_rows_of_one_value(C):
    """A row of one value has that value as its mean, whatever its bits: y is beta to the
    last bit, rstd that of eps, and dx that of a row whose xh is 0."""
    M = 200 if C < 1000 else 40
    x = full_mantissa(C, M)[:, None].expand(M, C).contiguous()
    gamma, beta, dy = rand(1, (C,), F32, 0.2, 1.0), rand(2, (C,), F32), rand(3, (M, C), F32)
    beta[: C // 2] = 0
    y, stats, dx = Out((M, C), F32), Out((M, 2), F32), Out((M, C), F32)
    dgamma, dbeta = Out((C,), F32), Out((C,), F32)
    dev = [t.to(DEV) for t in (x, gamma, beta, dy)]
    say("norm rows of one value", C)
    P.pyramid_layer_norm_forward(dev[0], dev[1], dev[2], y.t, stats.t)
    P.pyramid_layer_norm_backward(dev[0], dev[1], stats.t, dev[3], dx.t, dgamma.t, dbeta.t)
    assert torch.equal(stats.get()[:, 0], x[:, 0])
    assert torch.equal(y.get(), beta.expand(M, C))
    assert torch.equal(dgamma.get(), torch.zeros(C))
    rstd = torch.full((M, 1), 1e-5, dtype=torch.float64) ** -0.5
    a = (dy * gamma.double())
    want = rstd * (a - a.mean(1, keepdim=True))
    # a and its mean (64 serial additions at most), rstd: the root of eps, rounded itself
    near("dx", dx.get(), want, R.rounded(want, R.U * rstd * (6 * a.abs() + 70 * a.abs().mean(1, keepdim=True)), F32))


@pytest.mark.parametrize("offset,spread", [(1000.0, 1e-3), (1e6, 0.5), (-3e4, 0.02), (200.0, 1.0), (1e22, 1e16)])
@pytest.mark.parametrize("C", [16, 45, 1000, 5000])
def test_norm_far_above_the_spread(C, offset, spread):
    """fp32 rows far from zero, down to spreads of a few steps of their values: y is right to
    the bits of the differences, not of the values."""
    M = 60
    x = (rand(C, (M, C), F32).double() * spread + offset).float()
    gamma, beta = rand(1, (C,), F32, 0.2, 1.0), rand(2, (C,), F32)
    y, stats = Out((M, C), F32), Out((M, 2), F32)
    say("norm offset", C, offset, spread)
    P.pyramid_layer_norm_forward(x.to(DEV), gamma.to(DEV), beta.to(DEV), y.t, stats.t)
    ry, _, mean, rstd = R.norm_forward(x, gamma, beta, 1e-5, F32)
    near("mean", stats.get()[:, 0], mean[:, 0], 1.01 * R.U * mean[:, 0].abs())
    near("rstd", stats.get()[:, 1], rstd[:, 0], 40 * R.U * rstd[:, 0])
    # a difference from the mean is off by 3 U of itself (two subtractions, the mean's second
    # part) and U^2 of the mean; the variance by 70 U of itself, rstd by half of that and 4 U
    xh = (x.double() - mean) * rstd
    bound = (R.U * 44 * xh.abs() + 2 * R.U ** 2 * mean.abs() * rstd) * gamma.double().abs() + \
        R.U * (2 * ry.abs() + beta.double().abs())
    near("y", y.get(), ry, R.rounded(ry, bound, F32))


@pytest.mark.parametrize("C", [3, 45, 1000, 4099, 16384])
def test_norm_bf16_rows_of_one_value(C):
    x = full_mantissa(C, 60).to(BF16)[:, None].expand(60, C).contiguous()
    gamma, beta = rand(1, (C,), BF16, 0.2, 1.0), rand(2, (C,), BF16)
    beta[: C // 2] = 0
    y, stats = Out((60, C), BF16), Out((60, 2), F32)
    say("norm bf16 rows of one value", C)
    P.pyramid_layer_norm_forward(x.to(DEV), gamma.to(DEV), beta.to(DEV), y.t, stats.t)
    assert torch.equal(stats.get()[:, 0], x[:, 0].float()) and torch.equal(y.get(), beta.expand(60, C))


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("C", [3, 45, 64, 1000, 5000])
def test_norm_backward_of_huge_rows(C, ckpt):
    """Rows of one value whose mean times rstd passes fp32: channels that a row does not
    have do not get into its gradient."""
    M = 9
    x = torch.full((M, C), 2.0 ** 120)
    if not ckpt:        # blocks of codes span rows: one value in all of them
        x[1::2] *= -1.5
    gamma, dy = rand(1, (C,), F32, 0.2, 1.0), rand(2, (M, C), F32)
    dev = [t.to(DEV) for t in (x, gamma, dy)]
    y, stats, dx = Out((M, C), F32), Out((M, 2), F32), Out((M, C), F32)
    dgamma, dbeta = Out((C,), F32), Out((C,), F32)
    q, s = P.checkpoint8_empty(dev[0]) if ckpt else (None, None)
    say("norm huge rows", C, ckpt)
    P.pyramid_layer_norm_forward(dev[0], dev[1], dev[1], y.t, stats.t, q, s)
    if ckpt:        # the mean of the codes' values, so that their xh is 0
        stats.t[:, 0] = R.codes(x)[2][:, 0].float().to(DEV)
    P.pyramid_layer_norm_backward(dev[0] if q is None else q, dev[1], stats.t, dev[2], dx.t, dgamma.t, dbeta.t, xscale=s)
    assert torch.equal(dgamma.get(), torch.zeros(C))
    rstd = torch.full((M, 1), 1e-5, dtype=torch.float64) ** -0.5
    a = dy * gamma.double()
    want = rstd * (a - a.mean(1, keepdim=True))
    near("dx", dx.get(), want, R.rounded(want, R.U * rstd * (6 * a.abs() + 70 * a.abs().mean(1, keepdim=True)), F32))


def slow(shape, seed):
    """Waves along the steps, of other phases per channel: what a chunk inherits differs from
    one group of chunks to the next."""
    T, I = shape[1], shape[2]
    t, i = torch.arange(T, dtype=torch.float32)[:, None], torch.arange(I, dtype=torch.float32)[None]
    return torch.sin(t * (2 * 3.14159265 / 7000) + i * 0.7 + seed).expand(shape)


def scan_chain(B, T, I, dtype, cols, reverse=False, lengths=None, ckpt=False):
    """A chained scan of long memories, forward and backward, against the 64-bit form of the
    channels `cols`: all positions, hT and dh0."""
    g = rand(T + I, (B, T, I), dtype, 1.0, 7.5)
    u, dh = ((rand(T + I + k, (B, T, I), F32, 0.5) + slow((B, T, I), k)).to(dtype) for k in (1, 2))
    h0, dhT = rand(T + I + 3, (B, I), F32), rand(T + I + 4, (B, I), F32, 100.0)
    gd, ud, dhd, h0d, dhTd = (t.to(DEV) for t in (g, u, dh, h0, dhT))
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).to(DEV)
    h_, dg_, du_ = (Out((B, T, I), dtype) for _ in range(3))
    hT_, dh0_ = Out((B, I), F32), Out((B, I), F32)
    saved = torch.empty(P.pyramid_scan_saved_size(B, T, I), dtype=torch.uint8, device=DEV)
    P.pyramid_scan_forward(gd, ud, h_.t, reverse, ln, h0d, hT_.t, saved)
    gs = us = None
    gr, ur = g, u
    if ckpt:
        gk, gs = P.checkpoint8_empty(gd)
        uk, us = P.checkpoint8_empty(ud)
        P.pyramid_checkpoint8_pack(gd, gk, gs)
        P.pyramid_checkpoint8_pack(ud, uk, us)
        gd, ud = gk, uk
        gr, ur = R.codes(g)[2], R.codes(u)[2]
    P.pyramid_scan_backward(gd, ud, saved, dhd, dg_.t, du_.t, reverse, ln, dhTd, dh0_.t, gscale=gs, uscale=us)
    torch.cuda.synchronize()
    g, u, dh, gr, ur, h0, dhT = (t[..., cols].contiguous() for t in (g, u, dh, gr, ur, h0, dhT))
    h, e, hT, eT, before, eb = R.scan_forward(g, u, reverse, lengths, h0)
    near("h", h_.get()[..., cols], h, R.rounded(h, e, dtype))
    near("hT", hT_.get()[..., cols], hT, eT)
    if ckpt:
        before, eb = R.scan_forward(gr, ur, reverse, lengths, h0, run=(before, eb))[4:]
    (dg, eg), (du, eu), (dh0, e0) = R.scan_backward(gr, ur, before, eb, dh, reverse, lengths, dhT)
    near("dg", dg_.get()[..., cols], dg, R.rounded(dg, eg, dtype))
    near("du", du_.get()[..., cols], du, R.rounded(du, eu, dtype))
    near("dh0", dh0_.get()[..., cols], dh0, e0)


@DTYPES
@pytest.mark.parametrize("reverse", [False, True], ids=["fwd", "rev"])
@pytest.mark.parametrize("T,I,cols", [(20000, 3, [0, 1, 2]), (9000, 520, [0, 63, 64, 300, 511, 512, 519])],
                         ids=["groups-of-32", "groups-of-16"])
def test_scan_state_across_groups(T, I, cols, reverse, dtype):
    """States and their gradients from one group of chunks to the next, with groups of
    either size, in both directions."""
    say("scan groups", T, I, reverse, dtype)
    scan_chain(1, T, I, dtype, cols, reverse)


@DTYPES
@pytest.mark.parametrize("ckpt", [False, True], ids=["plain", "ckpt"])
@pytest.mark.parametrize("lengths", [None, [10000, 7777], [300, 10000]], ids=["even", "ragged", "ragged-short-first"])
def test_scan_chained_backward_of_eight_waves(lengths, ckpt, dtype):
    """More than 512 workgroups of sixteen waves: the backward takes eight."""
    B, I = (1, 1000) if lengths is None else (2, 500)
    assert -(-10000 // 256) * -(-B * I // 64) > 512
    say("scan eight waves", lengths, ckpt, dtype)
    scan_chain(B, 10000, I, dtype, [0, 63, 250, I - 1], lengths == [300, 10000], lengths, ckpt)


@DTYPES
@pytest.mark.parametrize("reverse", [False, True], ids=["fwd", "rev"])
@pytest.mark.parametrize("I", [64, 100, 192, 256])
def test_scan_ragged_codes_of_one_sequence(I, reverse, dtype):
    """Codes with lengths where a workgroup's columns are of one sequence."""
    say("scan ragged codes", I, reverse, dtype)
    scan_step(4, 290, I, dtype, reverse, [290, 0, 161, 288], ckpt=True, seed=I)


@pytest.mark.parametrize("M,C,dtype,ckpt", [
    ((1 << 21) + 300, 16, F32, True), ((1 << 22) + 700, 16, BF16, True),        # codes in lanes
    ((1 << 19) + 90, 45, F32, True), ((1 << 20) + 200, 45, BF16, True),         # codes through LDS
    ((1 << 20) + 77, 7, F32, True),                                             # codes by the pack kernel
    (8192 + 55, 2048, BF16, True), (8192 + 9, 1088, F32, True), (8192 + 20, 5000, F32, False),
    (8192 + 20, 4096, BF16, False), (8192 + 7, 9000, BF16, True), (8192 + 3, 16384, F32, False)],
    ids=lambda v: IDS.get(v, v) if isinstance(v, torch.dtype) else str(v))
def test_norm_workgroups_that_turn(M, C, dtype, ckpt):
    """More rows than the forward's 8192 workgroups (and the backward's 512) take at once:
    all rows, their codes and the weights' gradients."""
    gen = torch.Generator(device=DEV).manual_seed(M)
    x, dy = (torch.empty((M, C), dtype=dtype, device=DEV).normal_(k * 0.3, 0.8, generator=gen) for k in (1, 0))
    gamma, beta = rand(1, (C,), dtype, 0.2, 1.0).to(DEV), rand(2, (C,), dtype, 0.1).to(DEV)
    y, stats, dx = torch.empty_like(x), torch.empty((M, 2), device=DEV), torch.empty_like(x)
    dgamma, dbeta = torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    q, s = P.checkpoint8_empty(x) if ckpt else (None, None)
    say("norm turns", M, C, dtype, ckpt)
    P.pyramid_layer_norm_forward(x, gamma, beta, y, stats, q, s)
    P.pyramid_layer_norm_backward(x if q is None else q, gamma, stats, dy, dx, dgamma, dbeta, xscale=s)
    want = [torch.zeros(C, dtype=torch.float64, device=DEV) for _ in range(4)]
    step = 1 << 18 if C < 100 else 1 << 11      # rows, a multiple of 64: blocks of codes end with them
    for m in range(0, M, step):
        at = slice(m, m + step)
        ry, by, mean, rstd = R.norm_forward(x[at], gamma, beta, 1e-5, dtype)
        near("y", y[at], ry, by)
        kept = x[at]
        if ckpt:
            rq, rs, kept = R.codes(kept)
            assert torch.equal(q[at], rq) and torch.equal(s[m * C // 64:][:rs.numel()], rs)
        rdx, (dg, bg), (db, bb) = R.norm_backward(kept, mean, rstd, gamma, dy[at], dtype)
        near("dx", dx[at], *rdx)
        # the bounds of a part of the rows, with the chain of all of them
        more = (M - kept.shape[0]) / 256 * R.U
        xh = (kept.double() - mean) * rstd
        for t, v in zip(want, (dg, bg + more * (dy[at].double() * xh).abs().sum(0), db,
                               bb + more * dy[at].double().abs().sum(0))):
            t += v
    near("dgamma", dgamma, want[0], want[1])
    near("dbeta", dbeta, want[2], want[3])
