"""Edges of the block operators on the GPU: tensors that are given other memory between updates, more work than a
launch takes, arguments that are left out, numbers at the ends of fp32, and sums that are held in 64 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_1506_07452_amd as P
from paper_1506_07452_amd import network as net
from tests import block_ref as R
from tests.gpu_util import DEV, say
from tests.seq_ref import rounded
from tests.test_gpu_block import gn_case, poisoned
from tests.test_gpu_sequence import BF16, DTYPES, F32, near, rand

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------ AdamW

@pytest.mark.parametrize("bits", [32, 8])
def test_update_of_tensors_with_other_memory(bits):
    """Parameters and copies that are given other memory between updates, or replaced: as if nothing had happened, and the
    memory of before is left as it was."""
    say("adamw other memory", bits)
    sizes = [300, 17, 2049]
    p = [rand(k, (n,), F32).to(DEV) for k, n in enumerate(sizes)]
    grads = [[rand(10 * t + k, (n,), F32, 0.1).to(DEV) for k, n in enumerate(sizes)] for t in range(1, 4)]
    plain = P.AdamW([t.clone() for t in p], lr=1e-2, bits=bits, copies=[torch.zeros(n, dtype=BF16, device=DEV) for n in sizes], seed=9)
    moved = P.AdamW([t.clone() for t in p], lr=1e-2, bits=bits, copies=[torch.zeros(n, dtype=BF16, device=DEV) for n in sizes], seed=9)
    before = []
    for g in grads:
        plain.step(g)
        moved.step(g)
        for tensors in (moved.params, moved.copies):
            before += [(t, t.clone()) for t in (tensors[0].data, tensors[2])]
            tensors[0].data = tensors[0].data.clone()
            tensors[2] = tensors[2].clone()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(plain.params + plain.copies, moved.params + moved.copies))
    assert all(torch.equal(a, b) for a, b in zip(plain.m + plain.v, moved.m + moved.v))
    # all but the first update's went to memory of the update before
    assert all(torch.equal(a, b) for a, b in before)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [2.0 ** -149, 2.0 ** -130, 2.0 ** -126, 2.0 ** -100, 2.0 ** -50])
def test_update_with_a_tiny_eps(eps, bits):
    """An eps (fp32 numbers here, subnormal ones among them) whose reciprocal is no number: elements without a gradient so far
    only decay, others move by their quotient; gradients whose squares are 0 have eps alone below them."""
    say("adamw eps", eps, bits)
    n = 700
    p, g = rand(1, (n,), F32), rand(2, (n,), F32, 0.1)
    g[::3] = 0.0
    g[1::7] = 2.0 ** -80                # of the square an fp32 number holds nothing; over eps it is 2^69 at most
    p0 = p.to(DEV)
    opt = P.AdamW([p0], lr=1e-3, betas=(0.9, 0.99), eps=eps, weight_decay=0.1, bits=bits, seed=5)
    m, v = torch.zeros(n), torch.zeros(n)
    for t in (1, 2):
        new, bound, m, v = R.adamw(p, g, m, v, t, 1e-3, (0.9, 0.99), eps, 0.1)
        opt.step([g.to(DEV)])
        near("p", p0.cpu(), new, bound + 2.0 ** -23 * 1e-3 * 4)
        p = p0.cpu()
        if bits == 8:
            m, v = (x.cpu() for x in opt.moments()[0])


# ------------------------------------------------- more work than a launch takes

@pytest.mark.parametrize("N,G", [(1024, 4096), (1025, 4096), (513, 4100)])
def test_group_norm_of_groups_past_a_launch(N, G):
    """More groups than a launch of workgroups of 1024 has (fewer than 2^32 work items), a channel each: the last of them are
    in another launch, which the weights' gradients go with."""
    say("group norm of groups past a launch", N, G)
    gn_case(N, (2,), G, G, F32, seed=N)


def test_group_norm_of_volumes_past_a_launch():
    """As many volumes as there may be, each held by a workgroup of 1024."""
    N, V, period = 1 << 22, 1025, 64
    say("group norm of volumes past a launch")
    base, dbase = rand(1, (period, V, 1), BF16, 0.8, 0.3), rand(2, (period, V, 1), BF16, 0.3)
    gamma, beta = rand(3, (1,), BF16, 0.2, 1.0), rand(4, (1,), BF16, 0.3)
    x, dy = (b.to(DEV).repeat(N // period, 1, 1) for b in (base, dbase))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    stats, dg, db = torch.empty((N, 1, 2), device=DEV), torch.empty(1, device=DEV), torch.empty(1, device=DEV)
    P.pyramid_group_norm_forward(x, gamma.to(DEV), beta.to(DEV), y, 1, act="silu", stats=stats)
    P.pyramid_group_norm_backward(x, gamma.to(DEV), beta.to(DEV), stats, dy, dx, dg, db, 1, act="silu")
    torch.cuda.synchronize()
    for t in (y, dx, stats):
        rows = t.view(N // period, -1)
        assert all(bool((part == rows[0]).all()) for part in rows.split(1 << 13))
    (ry, ey), _, kept = R.group_norm(base, gamma, beta, 1, "silu", 1e-5)
    near("y", y[:period].cpu(), ry, rounded(ry, ey, BF16))
    (rx, ex), (rg, eg), (rb, eb) = R.group_norm_backward(kept, base, gamma, beta, dbase, 1, "silu")
    near("dx", dx[:period].cpu(), rx, rounded(rx, ex, BF16))
    times = N // period
    near("dgamma", dg.cpu(), rg * times, rounded(rg * times, eg * times, F32))
    near("dbeta", db.cpu(), rb * times, rounded(rb * times, eb * times, F32))


def test_conv_weights_past_a_launch():
    """So many channels that the sums of the weights' gradients have outputs in a second launch."""
    K, n = 4, 300
    I = (1 << 28) // (K + 1) + 5000
    say("convolution weights past a launch", I)
    gen = torch.Generator(device=DEV).manual_seed(1)

    def some(*shape, dtype=BF16):
        return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=gen)
    x, w, b, state, dy, dst = some(1, 1, I), some(I, K), some(I), some(1, K - 1, I), some(1, 1, I), some(1, K - 1, I, dtype=F32)
    dx, dw, db, before = torch.empty_like(x), torch.empty((I, K), device=DEV), torch.empty(I, device=DEV), torch.empty_like(dst)
    P.pyramid_causal_conv_backward(x, w, b, dy, dx, dw, db, act="silu", state=state, dstate_out=dst, dstate=before)
    # the first, those around the launches' border, the last
    for at in (0, (1 << 31) // 16 // (K + 1) - n // 2, I - n):
        c = slice(at, at + n)
        part = [t[..., c].cpu() for t in (x, b, state, dy, dst)]
        _, _, kept = R.conv_forward(part[0], w[c].cpu(), part[1], "silu", False, None, part[2])
        gx, gw, gb, gs = R.conv_backward(kept, w[c].cpu(), part[3], "silu", False, part[4])
        near("dx", dx[..., c].cpu(), gx[0], rounded(*gx, BF16))
        near("dw", dw[c].cpu(), *gw)
        near("db", db[c].cpu(), *gb)
        near("dstate", before[..., c].cpu(), *gs)


def test_scan_weights_past_a_launch():
    """The most channels of a scan: the sums of the weights' gradients have outputs in a second launch."""
    I, S, n = 1 << 24, 16, 200
    say("scan weights past a launch")
    gen = torch.Generator(device=DEV).manual_seed(2)

    def some(*shape, dtype=BF16):
        return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=gen)
    u, delta, dy = some(1, 1, I), some(1, 1, I), some(1, 1, I)
    Bm, Cm, h0, dhT = some(1, 1, S), some(1, 1, S), some(1, I, S, dtype=F32), some(1, I, S, dtype=F32)
    A, D, bias = some(I, S, dtype=F32).mul_(0.5).exp_().neg_(), some(I, dtype=F32), some(I, dtype=F32)
    saved = torch.empty(P.pyramid_selective_scan_saved_size(1, 1, I, S), dtype=torch.uint8, device=DEV)
    how = dict(D=D, delta_bias=bias, softplus=True)
    P.pyramid_selective_scan_forward(u, delta, A, Bm, Cm, torch.empty_like(u), h0=h0, saved=saved, **how)
    du, ddelta, dA, dB, dC = (torch.empty_like(t) for t in (u, delta, A, Bm, Cm))
    dD, dbias, dh0 = torch.empty_like(D), torch.empty_like(D), torch.empty_like(h0)
    P.pyramid_selective_scan_backward(u, delta, A, Bm, Cm, saved, dy, du, ddelta, dA, dB, dC, dD=dD, ddelta_bias=dbias, dhT=dhT, dh0=dh0,
                                      **how)
    # dA first, then dD and ddelta_bias: around the launches' border and in the last of all
    for at in (0, (1 << 31) // 16 // S - n // 2, I - n):
        c = slice(at, at + n)
        ref = R.Select(u[..., c].cpu(), delta[..., c].cpu(), A[c].cpu(), Bm.cpu(), Cm.cpu(), D[c].cpu(), None, bias[c].cpu(), True,
                       h0=h0[:, c].cpu())
        want = ref.backward(dy[..., c].cpu(), dhT[:, c].cpu())
        for name, got in (("dA", dA[c]), ("dD", dD[c]), ("ddelta_bias", dbias[c]), ("dh0", dh0[:, c])):
            near(name, got.cpu(), *want[name])
        for name, got in (("du", du), ("ddelta", ddelta)):
            near(name, got[..., c].cpu(), want[name][0], rounded(*want[name], BF16))


# ---------------------------------------------------- arguments that are left out

@pytest.mark.parametrize("left_out", [("conv_b",), ("D",), ("delta_bias",), ("conv_b", "D", "delta_bias")])
def test_sweep_without_biases(left_out):
    """A selective sweep's conv_b, D and delta_bias may be None: zeros, without a gradient."""
    say("sweep without", left_out)
    shape, I, S = (2, 3, 4, 9), 6, 4
    u, delta, z, dy = (rand(k, shape + (I,), F32, 0.5).to(DEV) for k in range(4))
    Bm, Cm = (rand(4 + k, shape + (S,), F32).to(DEV) for k in range(2))
    p = {"conv_w": rand(6, (I, 4), F32, 0.5), "conv_b": rand(7, (I,), F32, 0.2), "A": -torch.exp(rand(8, (I, S), F32, 0.5)),
         "D": rand(9, (I,), F32), "delta_bias": rand(10, (I,), F32, 0.5)}
    p = {k: torch.zeros_like(t).to(DEV) if k in left_out else t.to(DEV) for k, t in p.items()}
    y, kept = net.selective_forward(u, delta, z, Bm, Cm, p, "x", training=True)
    want = net.selective_backward(dy, kept, p)
    none = {k: None if k in left_out else t for k, t in p.items()}
    got_y, kept = net.selective_forward(u, delta, z, Bm, Cm, none, "x", training=True)
    got = net.selective_backward(dy, kept, none)
    assert torch.equal(y, got_y) and set(got) == set(want)
    for k, g in got.items():
        assert g is None if k in left_out else torch.equal(g, want[k]), k


# ------------------------------------------------------- numbers at the ends of fp32

@DTYPES
@pytest.mark.parametrize("B,T,I,S,lengths", [(4, 1, 7, 16, None), (5, 70, 18, 5, [0, 1, 33, 64, 70]), (3, 40, 17, 16, [40, 7, 0]),
                                             (2, 520, 16, 16, [520, 3]), (3, 90, 9, 40, [0, 90, 50]), (1, 1100, 33, 16, [500])])
@pytest.mark.parametrize("reverse", [False, True])
def test_scan_forgets(B, T, I, S, lengths, reverse, dtype):
    """States with A of minus infinity forget at once what was before a step, and keep what they have where a sequence has no
    steps; outputs and gradients as with an A of -1e25, whose decays are 0 and 1 as well."""
    say("select forgets", B, T, I, S, reverse, dtype)
    u, delta, z, dy = (poisoned(rand(k, (B, T, I), dtype), lengths) for k in range(4))
    Bm, Cm = (poisoned(rand(4 + k, (B, T, S), dtype), lengths) for k in range(2))
    h0, dhT, D, bias = rand(6, (B, I, S), F32), rand(7, (B, I, S), F32), rand(8, (I,), F32), rand(9, (I,), F32, 0.5, -2.0)
    A = -torch.exp(rand(10, (I, S), F32, 0.7))
    at_once = rand(11, (I, S), F32) > 0.5
    on = [None if t is None else t.to(DEV) for t in (u, delta, z, dy, Bm, Cm, h0, dhT, D, bias)]
    ud, dd, zd, dyd, Bd, Cd, h0d, dhTd, Dd, bd = on
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)

    def run(most):
        Ad = A.masked_fill(at_once, most).to(DEV)
        how = dict(D=Dd, z=zd, delta_bias=bd, softplus=True, reverse=reverse, lengths=ln)
        saved = torch.empty(P.pyramid_selective_scan_saved_size(B, T, I, S), dtype=torch.uint8, device=DEV)
        y, y2, hT, hT2 = torch.empty_like(ud), torch.empty_like(ud), torch.empty_like(h0d), torch.empty_like(h0d)
        P.pyramid_selective_scan_forward(ud, dd, Ad, Bd, Cd, y, h0=h0d, hT=hT, **how)
        P.pyramid_selective_scan_forward(ud, dd, Ad, Bd, Cd, y2, h0=h0d, hT=hT2, saved=saved, **how)
        g = dict(du=torch.empty_like(ud), ddelta=torch.empty_like(ud), dA=torch.empty_like(Ad), dB=torch.empty_like(Bd), dC=torch.empty_like(Bd),
                 dD=torch.empty_like(Dd), dz=torch.empty_like(ud), ddelta_bias=torch.empty_like(Dd), dh0=torch.empty_like(h0d))
        P.pyramid_selective_scan_backward(ud, dd, Ad, Bd, Cd, saved, dyd, dhT=dhTd, **g, **how)
        return dict(g, y=y, y2=y2, hT=hT, hT2=hT2)
    got, want = run(float("-inf")), run(-1e25)
    ref = R.Select(u, delta, A.masked_fill(at_once, -1e25), Bm, Cm, D, z, bias, True, reverse, lengths, h0)
    near("y", want["y"].cpu(), ref.y, rounded(ref.y, ref.ey, dtype))
    near("hT", want["hT"].cpu(), ref.hT, ref.ehT)
    for k, t in got.items():
        assert t.isfinite().all() and torch.equal(t, want[k]), k
    assert not got["dA"][at_once.to(DEV)].any()


# --------------------------------------------------------- sums in 64 bits
#
# Sums of N equal terms 1 + k 2^-23, whose last bits a running fp32 sum drops term by term once it is long
# enough, always in the same direction.  A kernel's bound counts the additions that it makes in fp32 before it goes on in 64
# bits, and the last rounding; one that added up a lane's terms in fp32 would be past it (`lost`).

def lost(c, n):
    """What a running fp32 sum of n terms c is off by, relative to it."""
    s = np.cumsum(np.full(n, c, np.float32), dtype=np.float32)[-1]
    return abs(float(s) / (n * c) - 1)


def equal_terms(name, got, c, n, additions, in_a_lane):
    """`got`: sums of n terms c with `additions` roundings to fp32, the last one among them, of each."""
    assert lost(c, in_a_lane) > 1.5 * additions * R.U, "these terms show nothing"
    want = torch.full_like(got, 1.0, dtype=torch.float64, device="cpu") * (n * c)
    near(name, got.cpu(), want, want * additions * R.U)


def test_group_norm_sums_in_64_bits():
    """Two rows in fp32, then 64 bits; a thread has 88 rows."""
    V, C, c = 1 << 24, 4, 1 + 15 * 2.0 ** -23
    say("group norm sums")
    x = torch.ones((1, V, C), device=DEV)
    x[:, ::2] = -1.0                        # mean 0, deviation 1
    one, zero = torch.ones(C, device=DEV), torch.zeros(C, device=DEV)
    y, stats, dg, db = torch.empty_like(x), torch.empty((1, 2, 2), device=DEV), torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    P.pyramid_group_norm_forward(x, one, zero, y, 2, stats=stats, eps=1e-30)
    assert torch.equal(y, x) and torch.equal(stats.cpu(), torch.tensor([[[0.0, 1.0]] * 2]))
    P.pyramid_group_norm_backward(x, one, zero, stats, torch.full_like(x, c), y, dg, db, 2)
    equal_terms("dbeta", db, c, V, 2, 88)
    assert not dg.any()
    P.pyramid_group_norm_backward(x, one, zero, stats, x * c, y, dg, db, 2)
    equal_terms("dgamma", dg, c, V, 2, 88)
    assert not db.any()


def test_scan_sums_in_64_bits():
    """16 steps of dA and 4 of dD and ddelta_bias in fp32 and a wave's share, then 64 bits; a wave has 1024 steps, a lane 256 of
    them."""
    T, I, S, c = 2048, 32768, 2, 1 + 63 * 2.0 ** -23
    say("scan sums")

    def full(v, *shape):
        return torch.full(shape, v, device=DEV)

    def run(u, B, dhT):
        """The gradients where all decays are 1, nothing is read out and the state before is 1."""
        one, A, D, Bm, Cm = full(1.0, 1, T, I), full(0.0, I, S), full(0.0, I), full(B, 1, T, S), full(0.0, 1, T, S)
        u, h0, dhT, y = full(u, 1, T, I), full(1.0, 1, I, S), full(dhT, 1, I, S), torch.empty((1, T, I), device=DEV)
        saved = torch.empty(P.pyramid_selective_scan_saved_size(1, T, I, S), dtype=torch.uint8, device=DEV)
        P.pyramid_selective_scan_forward(u, one, A, Bm, Cm, y, D=D, h0=h0, saved=saved)
        du, ddelta, dB, dC = torch.empty_like(u), torch.empty_like(u), torch.empty_like(Bm), torch.empty_like(Cm)
        dA, dD, db = torch.empty_like(A), torch.empty_like(D), torch.empty_like(D)
        P.pyramid_selective_scan_backward(u, one, A, Bm, Cm, saved, full(c, 1, T, I), du, ddelta, dA, dB, dC, D=D, dD=dD, ddelta_bias=db,
                                          dhT=dhT)
        return dA, dD, db
    # G = c and h = 1: dA sums c d; dp u = c
    dA, dD, _ = run(1.0, 0.0, c)
    equal_terms("dA", dA, c, T, 18, 1024)
    equal_terms("dD", dD, c, T, 6, 256)
    # u q with q = G summed over two states of 1/2
    _, _, db = run(c, 1.0, 0.5)
    equal_terms("ddelta_bias", db, c, T, 6, 256)


def test_conv_sums_in_64_bits():
    """Two runs of 32 steps a lane and 256 lanes of a workgroup in fp32, then 64 bits, however long a sequence is: with 512
    workgroups a lane of these would have 64 runs."""
    T, K, c = 1 << 28, 4, 1 + 511 * 2.0 ** -23
    say("convolution sums")
    x, dy = torch.ones((1, T, 1), device=DEV), torch.full((1, T, 1), c, device=DEV)
    dx, dw, db = torch.empty_like(x), torch.empty((1, K), device=DEV), torch.empty(1, device=DEV)
    P.pyramid_causal_conv_backward(x, torch.ones((1, K), device=DEV), torch.zeros(1, device=DEV), dy, dx, dw, db)
    for k in range(K):
        equal_terms("dw", dw[:, k], c, T - (K - 1) + k, 64 + 256 + 2, 2048)
    equal_terms("db", db, c, T, 64 + 256 + 2, 2048)
