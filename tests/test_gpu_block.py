"""The causal convolution, the selective scan, group norm with an activation and AdamW on
the GPU, against the plain 64-bit forms of tests/block_ref.py with their bounds."""
from __future__ import annotations

import pytest
import torch

import paper_1506_07452_amd as P
from tests import block_ref as R
from tests.gpu_util import DEV, say
from tests.seq_ref import TINY, rounded
from tests.test_gpu_sequence import BF16, DTYPES, F32, Out, near, rand

pytestmark = pytest.mark.gpu


def to_dev(*ts):
    return [None if t is None else t.to(DEV) for t in ts]


def sliced(t, before=3, after=5):
    """The tensor on the device as a slice of wider rows whose other elements are NaN."""
    wide = torch.full(t.shape[:-1] + (before + t.shape[-1] + after,), float("nan"), dtype=t.dtype, device=DEV)
    part = wide[..., before:before + t.shape[-1]]
    part.copy_(t)
    return part


def poisoned(t, lengths, reverse=False):
    """t with NaN at the steps that its sequences do not have."""
    t = t.clone()
    for b, n in enumerate(R.lengths_of(lengths, t.shape[0], t.shape[1])):
        t[b, n:] = float("nan")
    return t


# ------------------------------------------------------------------ convolution

def conv_case(B, T, I, K, dtype, act="silu", reverse=False, lengths=None, state=False, bias=True, slices=False, seed=0, stream=None):
    x, w = rand(seed, (B, T, I), dtype), rand(seed + 1, (I, K), dtype, 0.5)
    bv = rand(seed + 2, (I,), dtype, 0.2) if bias else None
    st = rand(seed + 3, (B, K - 1, I), dtype) if state else None
    dy, dst = rand(seed + 4, (B, T, I), dtype, 0.3), rand(seed + 5, (B, K - 1, I), F32, 0.3) if state else None
    xd = poisoned(x, lengths)
    xd = sliced(xd) if slices else xd.to(DEV)
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    wd, bd, std, dyd, dstd, lnd = to_dev(w, bv, st, poisoned(dy, lengths), dst, ln)
    y, dx, dw = Out((B, T, I), dtype), Out((B, T, I), dtype), Out((I, K), F32)
    db = Out((I,), F32) if bias else None
    after, before = (Out((B, K - 1, I), dtype), Out((B, K - 1, I), F32)) if state else (None, None)
    how = dict(act=act, reverse=reverse, lengths=lnd, state=std, stream=stream)
    P.pyramid_causal_conv_forward(xd, wd, bd, y.t, state_out=after.t if state else None, **how)
    P.pyramid_causal_conv_backward(xd, wd, bd, dyd, dx.t, dw.t, db.t if bias else None, dstate_out=dstd,
                                   dstate=before.t if state else None, **how)
    torch.cuda.synchronize()
    (ry, by), ra, kept = R.conv_forward(x, w, bv, act, reverse, lengths, st)
    near("y", y.get(), ry, rounded(ry, by, dtype))
    if state:
        assert torch.equal(after.get().double(), ra)
    gx, gw, gb, gs = R.conv_backward(kept, w, dy, act, reverse, dst)
    near("dx", dx.get(), gx[0], rounded(*gx, dtype))
    near("dw", dw.get(), *gw)
    if bias:
        near("db", db.get(), *gb)
    if state:
        near("dstate", before.get(), *gs)


@DTYPES
@pytest.mark.parametrize("K", [1, 2, 3, 4, 5, 6, 7, 8])
def test_conv_taps(K, dtype):
    say("conv taps", K, dtype)
    conv_case(2, 37, 19, K, dtype, state=K > 1, seed=K)


@DTYPES
@pytest.mark.parametrize("B,T,I", [(1, 1, 1), (3, 1, 2048), (1, 2, 5), (2, 3, 3), (1, 8, 4), (2, 9, 17), (1, 31, 64), (1, 32, 65),
                                   (1, 33, 7), (5, 65, 16), (2, 300, 8), (1, 1000, 1), (40, 7, 6), (1, 4, 4099)])
def test_conv_sizes(B, T, I, dtype):
    say("conv sizes", B, T, I, dtype)
    conv_case(B, T, I, 4, dtype, seed=T)
    conv_case(B, T, I, 4, dtype, act="none", reverse=True, state=True, bias=False, slices=True, seed=T + 1)


@DTYPES
@pytest.mark.parametrize("reverse", [False, True])
def test_conv_lengths(reverse, dtype):
    """Sequences of nothing, less than the taps, all; NaN where there are no steps."""
    say("conv lengths", reverse, dtype)
    conv_case(9, 70, 21, 4, dtype, reverse=reverse, lengths=[0, 1, 2, 3, 4, 33, 69, 70, 99], state=True, slices=True)
    conv_case(3, 70, 21, 8, dtype, reverse=reverse, lengths=[-5, 5, 64], state=True)


@DTYPES
def test_conv_state_in_place(dtype):
    """Single steps with the state updated where it is give what one call over all gives."""
    B, T, I, K = 3, 11, 33, 4
    x, w, b = rand(1, (B, T, I), dtype).to(DEV), rand(2, (I, K), dtype).to(DEV), rand(3, (I,), dtype).to(DEV)
    whole, steps = torch.empty_like(x), torch.empty_like(x)
    state = torch.zeros((B, K - 1, I), dtype=dtype, device=DEV)
    P.pyramid_causal_conv_forward(x, w, b, whole, act="silu")
    for t in range(T):
        y = torch.empty((B, 1, I), dtype=dtype, device=DEV)
        P.pyramid_causal_conv_forward(x[:, t:t + 1], w, b, y, act="silu", state=state, state_out=state)
        steps[:, t:t + 1] = y
    assert torch.equal(steps, whole) and torch.equal(state, x[:, -3:])


# --------------------------------------------------------------- selective scan

def scan_case(B, T, I, S, dtype, reverse=False, lengths=None, state=False, gate=True, softplus=True, skip=True, slices=False,
              seed=0, stream=None, shift=-3.0, want=("dD", "ddelta_bias", "dh0")):
    u, delta = rand(seed, (B, T, I), dtype), rand(seed + 1, (B, T, I), dtype, 0.7)
    if not softplus:
        delta = delta.abs() * 0.1
    dbias = rand(seed + 2, (I,), F32, 1.0, shift) if softplus else None
    A = -torch.exp(rand(seed + 3, (I, S), F32, 0.7, 0.5))
    Bm, Cm = rand(seed + 4, (B, T, S), dtype), rand(seed + 5, (B, T, S), dtype)
    D = rand(seed + 6, (I,), F32) if skip else None
    z = rand(seed + 7, (B, T, I), dtype, 1.5) if gate else None
    h0 = rand(seed + 8, (B, I, S), F32) if state else None
    dy, dhT = rand(seed + 9, (B, T, I), dtype, 0.3), rand(seed + 10, (B, I, S), F32, 0.3) if state else None
    ref = R.Select(u, delta, A, Bm, Cm, D, z, dbias, softplus, reverse, lengths, h0)
    grads = ref.backward(dy, dhT)

    def put(t, cut):
        if t is None:
            return None
        t = poisoned(t, lengths)
        return sliced(t) if slices and cut else t.to(DEV)

    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    ud, dd, Bd, Cd, zd, dyd = put(u, 1), put(delta, 1), put(Bm, 1), put(Cm, 1), put(z, 1), put(dy, 0)
    Ad, Dd, biasd, h0d, dhTd, lnd = to_dev(A, D, dbias, h0, dhT, ln)
    how = dict(D=Dd, z=zd, delta_bias=biasd, softplus=softplus, reverse=reverse, lengths=lnd, stream=stream)
    saved = torch.full((P.pyramid_selective_scan_saved_size(B, T, I, S),), 0x7f, dtype=torch.uint8, device=DEV)
    first, y, hT = Out((B, T, I), dtype), Out((B, T, I), dtype), Out((B, I, S), F32)
    P.pyramid_selective_scan_forward(ud, dd, Ad, Bd, Cd, first.t, h0=h0d, **how)
    P.pyramid_selective_scan_forward(ud, dd, Ad, Bd, Cd, y.t, h0=h0d, hT=hT.t, saved=saved, **how)
    o = {k: Out((B, T, I), dtype) for k in ("du", "ddelta") + (("dz",) if gate else ())}
    o.update(dB=Out((B, T, S), dtype), dC=Out((B, T, S), dtype), dA=Out((I, S), F32))
    o.update({k: Out((B, I, S) if k == "dh0" else (I,), F32) for k in want})
    g = {k: v.t for k, v in o.items()}
    P.pyramid_selective_scan_backward(ud, dd, Ad, Bd, Cd, saved, dyd, dhT=dhTd, **g, **how)
    torch.cuda.synchronize()
    near("y", y.get(), ref.y, rounded(ref.y, ref.ey, dtype))
    if T > 1:
        assert torch.equal(first.get(), y.get()), "y of inference"
    else:
        near("y of inference", first.get(), ref.y, rounded(ref.y, ref.ey, dtype))
    near("hT", hT.get(), ref.hT, ref.ehT)
    for k, out in o.items():
        v, e = grads[k]
        near(k, out.get(), v, rounded(v, e, F32 if k in ("dA", "dD", "ddelta_bias", "dh0") else dtype))


@DTYPES
@pytest.mark.parametrize("S", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 24, 32, 33, 48, 63, 64])
def test_scan_states(S, dtype):
    say("select states", S, dtype)
    scan_case(2, 70, 19, S, dtype, state=True, seed=S)


@DTYPES
@pytest.mark.parametrize("T", [1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300])
def test_scan_lengths_of_time(T, dtype):
    say("select steps", T, dtype)
    scan_case(2, T, 17, 16, dtype, seed=T)
    scan_case(1, T, 5, 3, dtype, state=True, reverse=True, seed=T + 1)


@DTYPES
@pytest.mark.parametrize("B,I", [(1, 1), (1, 2), (3, 15), (2, 16), (5, 33), (1, 64), (1, 130), (33, 4), (2, 257)])
def test_scan_columns(B, I, dtype):
    say("select columns", B, I, dtype)
    scan_case(B, 40, I, 8, dtype, seed=I, slices=True)


@DTYPES
@pytest.mark.parametrize("gate,softplus,skip", [(False, True, True), (True, False, True), (True, True, False), (False, False, False)])
def test_scan_without(gate, softplus, skip, dtype):
    say("select without", gate, softplus, skip, dtype)
    scan_case(2, 50, 20, 16, dtype, gate=gate, softplus=softplus, skip=skip, reverse=True, want=())


@DTYPES
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("S", [5, 16, 40])
def test_scan_ragged(S, reverse, dtype):
    """Sequences of nothing, of a part of a tile, all; NaN where there are no steps."""
    say("select ragged", S, reverse, dtype)
    scan_case(8, 130, 18, S, dtype, reverse=reverse, lengths=[0, 1, 17, 64, 65, 129, 130, 500], state=True, slices=True, seed=S)


@DTYPES
@pytest.mark.parametrize("B,T,I,S", [(1, 1100, 33, 16), (2, 520, 16, 4), (1, 700, 7, 20), (1, 300, 9, 64)])
@pytest.mark.parametrize("reverse", [False, True])
def test_scan_chunks(B, T, I, S, reverse, dtype):
    """Long sequences of few channels are cut into chunks that run at the same time."""
    say("select chunks", B, T, I, S, reverse, dtype)
    scan_case(B, T, I, S, dtype, reverse=reverse, state=True, seed=T)
    scan_case(B, T, I, S, dtype, reverse=reverse, state=True, seed=T + 1, lengths=[T - 70] + [3] * (B - 1))


def test_scan_many_jobs():
    """More sequences than a backward has workgroups for at once."""
    say("select jobs")
    scan_case(1100, 9, 3, 2, F32, seed=5)


def test_scan_softplus_ends():
    """Steps far below and above softplus's bend keep their relative accuracy."""
    say("select softplus")
    for shift in (-12.0, -7.0, 8.0, 30.0):
        scan_case(2, 33, 18, 4, F32, shift=shift, gate=False, seed=int(shift) + 50)


@DTYPES
@pytest.mark.parametrize("S", [1, 4, 6, 16, 30, 64])
def test_scan_token(S, dtype):
    """Single steps with the state updated where it is follow one call over all of them."""
    say("select token", S, dtype)
    B, T, I = 3, 6, 21
    u, delta, z = (rand(k, (B, T, I), dtype).to(DEV) for k in range(3))
    Bm, Cm = (rand(k, (B, T, S), dtype).to(DEV) for k in (4, 5))
    A, D, bias = to_dev(-torch.exp(rand(6, (I, S), F32)), rand(7, (I,), F32), rand(8, (I,), F32, 1.0, -2.0))
    h0 = rand(9, (B, I, S), F32)
    ref = R.Select(*(t.cpu() for t in (u, delta, A, Bm, Cm, D, z, bias)), softplus=True, h0=h0)
    h = h0.to(DEV)
    steps = Out((B, T, I), dtype)
    for t in range(T):
        y = torch.empty((B, 1, I), dtype=dtype, device=DEV)
        P.pyramid_selective_scan_forward(*(v[:, t:t + 1] if v.dim() == 3 else v for v in (u, delta, A, Bm, Cm)), y, D=D,
                                         z=z[:, t:t + 1], delta_bias=bias, softplus=True, h0=h, hT=h)
        steps.t[:, t:t + 1] = y
    near("y", steps.get(), ref.y, rounded(ref.y, ref.ey, dtype))
    near("hT", h.cpu(), ref.hT, ref.ehT)
    # a sequence without the step keeps its state
    kept = h.clone()
    y = torch.full((B, 1, I), 7.0, dtype=dtype, device=DEV)
    P.pyramid_selective_scan_forward(u[:, :1], delta[:, :1], A, Bm[:, :1], Cm[:, :1], y, h0=h, hT=h, softplus=True,
                                     lengths=torch.tensor([1, 0, 1], dtype=torch.int32, device=DEV))
    assert torch.equal(h[1], kept[1]) and not torch.equal(h[0], kept[0]) and (y[1] == 0).all()


def test_scan_state_in_place_of_chunks():
    """hT may be h0 and dh0 dhT also where chunks of a sequence run at the same time."""
    B, T, I, S = 1, 1500, 18, 16
    u, delta, dy = (rand(k, (B, T, I), F32).to(DEV) for k in range(3))
    Bm, Cm = (rand(k, (B, T, S), F32).to(DEV) for k in (4, 5))
    A = -torch.exp(rand(6, (I, S), F32)).to(DEV)
    h0, dhT = (rand(k, (B, I, S), F32).to(DEV) for k in (7, 8))

    def run(hT, dh0, h0, dhT):
        y, du, dd = (torch.empty_like(u) for _ in range(3))
        dA, dB, dC = torch.empty_like(A), torch.empty_like(Bm), torch.empty_like(Cm)
        saved = torch.empty(P.pyramid_selective_scan_saved_size(B, T, I, S), dtype=torch.uint8, device=DEV)
        P.pyramid_selective_scan_forward(u, delta, A, Bm, Cm, y, softplus=True, h0=h0, hT=hT, saved=saved)
        P.pyramid_selective_scan_backward(u, delta, A, Bm, Cm, saved, dy, du, dd, dA, dB, dC, softplus=True, dhT=dhT, dh0=dh0)
        return [y, hT, du, dd, dA, dB, dC, dh0]

    want = run(torch.empty_like(h0), torch.empty_like(dhT), h0, dhT)
    a, b = h0.clone(), dhT.clone()
    got = run(a, b, a, b)
    assert all(torch.equal(x, y) for x, y in zip(want, got))


# ------------------------------------------------------------------- group norm

def gn_case(N, shape, C, G, dtype, act="silu", want_dx=True, seed=0, x=None, stream=None):
    full = (N,) + shape + (C,)
    x = rand(seed, full, dtype, 0.8, 0.3) if x is None else x
    gamma, beta, dy = rand(seed + 1, (C,), dtype, 0.2, 1.0), rand(seed + 2, (C,), dtype, 0.3), rand(seed + 3, full, dtype, 0.3)
    xd, gd, bd, dyd = to_dev(x, gamma, beta, dy)
    y, stats, dx = Out(full, dtype), Out((N, G, 2), F32), Out(full, dtype)
    dg, db = Out((C,), F32), Out((C,), F32)
    P.pyramid_group_norm_forward(xd, gd, bd, y.t, G, act=act, stats=stats.t, stream=stream)
    P.pyramid_group_norm_backward(xd, gd, bd, stats.t, dyd, dx.t if want_dx else None, dg.t, db.t, G, act=act, stream=stream)
    torch.cuda.synchronize()
    (ry, ey), (mean, rstd), kept = R.group_norm(x, gamma, beta, G, act, 1e-5)
    near("y", y.get(), ry, rounded(ry, ey, dtype))
    near("mean", stats.get()[..., 0], mean, 2 * R.U * mean.abs() + TINY + 2.0 ** -50 * x.double().abs().max())
    near("rstd", stats.get()[..., 1], rstd, rstd * (2 * R.U + 2.0 ** -48 * (1 + mean ** 2 * rstd ** 2)))
    (rx, ex), (rg, eg), (rb, eb) = R.group_norm_backward(kept, x, gamma, beta, dy, G, act)
    if want_dx:
        near("dx", dx.get(), rx, rounded(rx, ex, dtype))
    near("dgamma", dg.get(), rg, rounded(rg, eg, F32))
    near("dbeta", db.get(), rb, rounded(rb, eb, F32))


@DTYPES
@pytest.mark.parametrize("C,G", [(1, 1), (2, 1), (3, 3), (4, 2), (7, 1), (8, 8), (15, 5), (16, 4), (17, 17), (25, 5), (32, 8), (45, 9), (64, 8),
                                 (65, 13), (90, 3), (128, 32), (250, 10), (333, 111), (1024, 32), (1030, 103), (2048, 16), (2050, 2), (4100, 41),
                                 (9000, 9), (16384, 64)])
def test_group_norm_channels(C, G, dtype):
    say("group norm", C, G, dtype)
    gn_case(2, (5,), C, G, dtype, seed=C)
    gn_case(1, (37,), C, G, dtype, act="none", seed=C + 1)


@DTYPES
@pytest.mark.parametrize("N,shape", [(1, (1,)), (1, ()), (700, ()), (300, (2,)), (1, (255,)), (3, (256,)), (1, (4, 8, 16)), (2, (1000,)), (1, (4096,)),
                                     (2, (13, 17, 19)), (1, (20000,)), (5, (9001,))])
def test_group_norm_volumes(N, shape, dtype):
    say("group norm volumes", N, shape, dtype)
    gn_case(N, shape, 16, 4, dtype, seed=N)
    gn_case(N, shape, 45, 5, dtype, seed=N + 1, want_dx=N % 2 == 0)


@DTYPES
def test_group_norm_far_from_zero(dtype):
    """Groups of one value, far above their spread, and with a first voxel unlike the others."""
    say("group norm far", dtype)
    for V in (50, 30000):
        x = torch.full((1, V, 8), 1000.0)
        gn_case(1, (V,), 8, 2, dtype, x=x.to(dtype))
        if dtype == F32:
            x = 1000.0 + rand(1, (1, V, 8), F32)
            gn_case(1, (V,), 8, 2, dtype, x=x)
            x[:, 0] = 0.0
            gn_case(1, (V,), 8, 4, dtype, x=x)


@DTYPES
def test_group_norm_not_finite(dtype):
    """A group with an infinity or a NaN is NaN, the others are as they are."""
    for V in (40, 20000):
        x = rand(1, (2, V, 16), dtype).to(DEV)
        gamma, beta = torch.ones(16, dtype=dtype, device=DEV), torch.zeros(16, dtype=dtype, device=DEV)
        want, got = torch.empty_like(x), torch.empty_like(x)
        P.pyramid_group_norm_forward(x, gamma, beta, want, 4)
        x[0, 3, 5], x[1, 7, 15] = float("nan"), float("inf")
        P.pyramid_group_norm_forward(x, gamma, beta, got, 4)
        bad = torch.zeros((2, V, 16), dtype=torch.bool, device=DEV)
        bad[0, :, 4:8] = bad[1, :, 12:] = True
        assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], want[~bad])


# ------------------------------------------------------------------------ AdamW

SIZES = [1, 3, 4, 5, 255, 256, 257, 1000, 2048, 2049, 7777]
HOW = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-6)


def adam_inputs(sizes, gdtype, seed=0):
    p, g = [rand(seed + k, (n,), F32) for k, n in enumerate(sizes)], [rand(seed + 100 + k, (n,), gdtype, 0.1) for k, n in enumerate(sizes)]
    return p, g


@DTYPES
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_steps(bits, dtype):
    """Three updates: parameters within their bound, moments (codes and scales of them) exactly."""
    say("adamw", bits, dtype)
    p, _ = adam_inputs(SIZES, dtype)
    decay = [0.01 * (k % 3) for k in range(len(SIZES))]
    pd = [Out(t.shape, F32) for t in p]
    for o, t in zip(pd, p):
        o.t.copy_(t)
    copies = [Out(t.shape, BF16) for t in p]
    opt = P.AdamW([o.t for o in pd], weight_decay=decay, bits=bits, copies=[c.t for c in copies], seed=12345, **HOW)
    m, v = ([torch.zeros(n) for n in SIZES] for _ in range(2))
    scale = torch.tensor([0.75], device=DEV)
    for t in range(1, 4):
        _, g = adam_inputs(SIZES, dtype, seed=1000 * t)
        if t == 2:
            g[4][:40] = 0.0
        opt.step(to_dev(*g), grad_scale=scale if t > 1 else None)
        torch.cuda.synchronize()
        assert opt.t == t
        for k, n in enumerate(SIZES):
            new, bound, m[k], v[k] = R.adamw(p[k], g[k], m[k], v[k], t, HOW["lr"], HOW["betas"], HOW["eps"], decay[k],
                                             0.75 if t > 1 else 1.0)
            # lr, eps and the decays are fp32 numbers in the kernel
            near("p", pd[k].get(), new, bound + 2.0 ** -23 * HOW["lr"] * 4)
            p[k] = pd[k].get()
            assert torch.equal(copies[k].get(), p[k].to(BF16))
            if bits == 32:
                assert torch.equal(opt.m[k].cpu(), m[k]) and torch.equal(opt.v[k].cpu(), v[k])
            else:
                lo, hi = R.halves_of(n, 12345, t, k)
                for name, x, got, scales, half, E in (("m", m[k], opt.m[k], opt.mscale[k], lo, 4), ("v", v[k], opt.v[k], opt.vscale[k], hi, 5)):
                    codes, want = R.narrow(x, E, half)
                    assert torch.equal(scales.cpu(), want), name
                    assert torch.equal(got.cpu(), codes), name
                m[k], v[k] = R.wide(opt.m[k].cpu(), opt.mscale[k].cpu(), 4), R.wide(opt.v[k].cpu(), opt.vscale[k].cpu(), 5)
        for k, (mm, vv) in enumerate(opt.moments()):
            assert torch.equal(mm.cpu(), m[k]) and torch.equal(vv.cpu(), v[k])


def test_adamw_many_tensors():
    """More tensors than a launch takes, empty ones and ones without a gradient among them."""
    say("adamw many")
    sizes = [(7 * k) % 301 for k in range(131)]
    p, g = adam_inputs(sizes, F32)
    pd, gd = to_dev(*p), to_dev(*g)
    gd[5] = gd[64] = None
    for bits in (32, 8):
        mine = [t.clone() for t in pd]
        opt = P.AdamW(mine, bits=bits, **HOW)
        opt.step(gd)
        for k, n in enumerate(sizes):
            if gd[k] is None:
                assert torch.equal(mine[k], pd[k]) and not opt.m[k].any()
            elif n:
                new, bound, m, v = R.adamw(p[k], g[k], torch.zeros(n), torch.zeros(n), 1, HOW["lr"], HOW["betas"], HOW["eps"], 0.01)
                near("p", mine[k].cpu(), new, bound + 2.0 ** -23 * HOW["lr"] * 4)
                if bits == 8:
                    assert torch.equal(opt.m[k].cpu(), R.narrow(m, 4, R.halves_of(n, 0, 1, k)[0])[0])


def test_adamw_rounding_is_unbiased():
    """A second moment that moves by 1e-3 of itself a step follows its gradients in 8 bits.  With b2 = 0.99 and
    constant gradients v_t = g^2 (1 - 0.99^t); a code is off by at most an eighth of the value each step, of which
    b2 keeps 0.99: the variance of 4096 such values adds up to (1/8)^2 / 4 / (1 - 0.99^2) of v^2 at most, a deviation of 0.45, of their
    mean 0.007.  Five of those."""
    n = 4096
    g = torch.full((n,), 0.5, device=DEV)
    g[::256] = 1.0          # the largest of each block
    opt = P.AdamW([torch.zeros(n, device=DEV)], lr=0.0, betas=(0.9, 0.99), bits=8)
    for _ in range(200):
        opt.step([g])
    m, v = opt.moments()[0]
    keep = torch.ones(n, dtype=torch.bool, device=DEV)
    keep[::256] = False
    want = 0.25 * (1 - 0.99 ** 200)
    assert abs(float(v[keep].double().mean()) / want - 1) < 0.035
    assert abs(float(m[keep].double().mean()) / 0.5 - 1) < 0.035


def test_adamw_not_finite():
    """A block with a NaN or an infinity becomes NaN; the others do not."""
    g = rand(1, (1024,), F32).to(DEV)
    g[3], g[600] = float("nan"), float("inf")
    p = torch.zeros(1024, device=DEV)
    opt = P.AdamW([p], bits=8)
    opt.step([g])
    m, v = opt.moments()[0]
    for k, bad in enumerate((True, False, True, False)):
        b = slice(256 * k, 256 * k + 256)
        assert torch.isnan(m[b]).all() == bad and torch.isnan(v[b]).all() == bad
        assert not bad or torch.isnan(opt.mscale[0][k])


def test_adamw_state_goes_on():
    """state() of one optimiser taken up by another goes on as the first would."""
    for bits in (32, 8):
        p, _ = adam_inputs([300, 17], F32)
        a, b = ([t.to(DEV) for t in p] for _ in range(2))
        one = P.AdamW(a, bits=bits, seed=3)
        gs = [to_dev(*adam_inputs([300, 17], F32, seed=s)[1]) for s in range(4)]
        for g in gs:
            one.step(g)
        two = P.AdamW(b, bits=bits, seed=3)
        two.step(gs[0])
        two.step(gs[1])
        three = P.AdamW(b, bits=bits, seed=3, state=two.state())
        three.step(gs[2])
        three.step(gs[3])
        assert three.t == 4 and all(torch.equal(x, y) for x, y in zip(a, b)) and all(
            torch.equal(x, y) for x, y in zip(one.m + one.v, three.m + three.v))
