"""Refusals of the causal convolution, selective scan, group norm and AdamW entry points (C ABI, no GPU:
validation comes before any HIP call), and the 64-bit forms that the GPU tests use, against autograd,
differences and counts."""
from __future__ import annotations

import ctypes

import pytest
import torch

import paper_1506_07452_amd as P
from tests import block_ref as R

FAKE = ctypes.c_void_p(0x10000)      # aligned, never dereferenced
ODD = ctypes.c_void_p(0x10001)
BIG = 1 << 50
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    return P.load()


def conv_fwd(lib, B=2, T=5, I=8, K=4, dtype=0, act=1, reverse=0, x=FAKE, px=0, w=FAKE, bias=None, lengths=None, state=None,
             y=FAKE, out=None):
    return lib.pyramid_causal_conv_forward(B, T, I, K, dtype, act, reverse, x, px, w, bias, lengths, state, y, out, None)


def conv_bwd(lib, B=2, T=5, I=8, K=4, dtype=0, act=1, reverse=0, x=FAKE, px=0, w=FAKE, bias=None, lengths=None, state=None,
             dy=FAKE, dso=None, dx=FAKE, dw=FAKE, db=None, ds=None, ws=FAKE, nbytes=BIG):
    return lib.pyramid_causal_conv_backward(B, T, I, K, dtype, act, reverse, x, px, w, bias, lengths, state, dy, dso, dx, dw,
                                            db, ds, ws, nbytes, None)


def test_conv_refusals(lib):
    common = [dict(B=0), dict(T=0), dict(I=0), dict(K=0), dict(dtype=2), dict(act=2), dict(act=-1), dict(reverse=2), dict(x=None),
              dict(w=None), dict(px=7), dict(px=-1), dict(px=1 << 62), dict(x=ODD), dict(bias=ODD), dict(lengths=ODD), dict(state=ODD)]
    for bad in common + [dict(y=None), dict(y=ODD), dict(out=ODD)]:
        assert conv_fwd(lib, **bad) == -1, bad
    for bad in common + [dict(dy=None), dict(dx=None), dict(dw=None), dict(ws=None), dict(dso=ODD), dict(dw=ODD), dict(db=ODD),
                         dict(ds=ODD), dict(ws=ODD)]:
        assert conv_bwd(lib, **bad) == -1, bad
    for bad in (dict(K=9), dict(T=(1 << 31) + 1), dict(B=1 << 20, T=1 << 20), dict(I=1 << 31)):
        assert conv_fwd(lib, **bad) == -2 and conv_bwd(lib, **bad) == -2, bad
    need = P.pyramid_causal_conv_workspace_size(2, 5, 8, 4)
    assert need > 0 and conv_bwd(lib, nbytes=need - 1) == -3
    for bad in ((0, 5, 8, 4), (2, 5, 8, 9), (2, 1 << 40, 8, 4)):
        assert P.pyramid_causal_conv_workspace_size(*bad) == 0


SELECT = dict(B=2, T=5, I=8, S=16, dtype=0, reverse=0, softplus=1, u=FAKE, pu=0, delta=FAKE, pd=0, A=FAKE, Bm=FAKE, pB=0, Cm=FAKE,
              pC=0, D=None, z=None, pz=0, bias=None, lengths=None)


def sel_fwd(lib, h0=None, y=FAKE, hT=None, saved=None, ws=FAKE, nbytes=BIG, **kw):
    return lib.pyramid_selective_scan_forward(*dict(SELECT, **kw).values(), h0, y, hT, saved, ws, nbytes, None)


def sel_bwd(lib, saved=FAKE, dy=FAKE, dhT=None, du=FAKE, ddelta=FAKE, dA=FAKE, dB=FAKE, dC=FAKE, dD=None, dz=None, ddb=None,
            dh0=None, ws=FAKE, nbytes=BIG, **kw):
    return lib.pyramid_selective_scan_backward(*dict(SELECT, **kw).values(), saved, dy, dhT, du, ddelta, dA, dB, dC, dD, dz, ddb,
                                               dh0, ws, nbytes, None)


def test_selective_scan_refusals(lib):
    common = [dict(B=0), dict(T=-1), dict(I=0), dict(S=0), dict(dtype=3), dict(reverse=-1), dict(softplus=2), dict(u=None), dict(delta=None),
              dict(A=None), dict(Bm=None), dict(Cm=None), dict(pu=7), dict(pd=-8), dict(pz=3), dict(pB=15), dict(pC=1), dict(pB=1 << 60),
              dict(u=ODD), dict(A=ODD), dict(Bm=ODD), dict(D=ODD), dict(bias=ODD), dict(lengths=ODD), dict(saved=ODD), dict(ws=ODD), dict(ws=None)]
    for bad in common + [dict(y=None), dict(y=ODD), dict(h0=ODD), dict(hT=ODD), dict(z=ODD)]:
        assert sel_fwd(lib, **bad) == -1, bad
    for bad in common + [dict(saved=None), dict(dy=None), dict(du=None), dict(ddelta=None), dict(dA=None), dict(dB=None), dict(dC=None),
                         dict(dz=FAKE), dict(z=FAKE), dict(dhT=ODD), dict(dh0=ODD), dict(dA=ODD), dict(dC=ODD), dict(dD=ODD), dict(ddb=ODD)]:
        assert sel_bwd(lib, **bad) == -1, bad
    for bad in (dict(S=65), dict(T=(1 << 31) + 1), dict(B=1 << 30, I=1 << 30), dict(B=1 << 23, I=1), dict(B=1 << 20, T=1 << 20)):
        assert sel_fwd(lib, **bad) == -2 and sel_bwd(lib, **bad) == -2, bad
    for backward, call in ((0, sel_fwd), (1, sel_bwd)):
        need = P.pyramid_selective_scan_workspace_size(2, 5, 8, 16, backward)
        assert need > 0 and call(lib, nbytes=need - 1) == -3
    for bad in ((0, 5, 8, 16), (2, 5, 8, 65), (2, 5, 1 << 40, 16)):
        assert P.pyramid_selective_scan_workspace_size(*bad) == 0 and P.pyramid_selective_scan_saved_size(*bad) == 0
    assert lib.pyramid_selective_scan_workspace_size(2, 5, 8, 16, 2) == 0
    # a state for each 16 positions
    for S in (1, 16, 17, 64):
        assert P.pyramid_selective_scan_saved_size(3, 33, 16, S) == 3 * 3 * 16 * S * 4 + -(3 * 3 * 16 * S * 4) % 256


def gn_fwd(lib, N=2, V=5, C=8, G=4, dtype=0, act=1, eps=1e-5, x=FAKE, gamma=FAKE, beta=FAKE, y=FAKE, stats=None, ws=FAKE, nbytes=BIG):
    return lib.pyramid_group_norm_forward(N, V, C, G, dtype, act, eps, x, gamma, beta, y, stats, ws, nbytes, None)


def gn_bwd(lib, N=2, V=5, C=8, G=4, dtype=0, act=1, x=FAKE, gamma=FAKE, beta=FAKE, stats=FAKE, dy=FAKE, dx=FAKE, dgamma=FAKE, dbeta=FAKE,
           ws=FAKE, nbytes=BIG):
    return lib.pyramid_group_norm_backward(N, V, C, G, dtype, act, x, gamma, beta, stats, dy, dx, dgamma, dbeta, ws, nbytes, None)


def test_group_norm_refusals(lib):
    common = [dict(N=0), dict(V=0), dict(C=0), dict(G=0), dict(G=3), dict(G=16), dict(dtype=2), dict(act=2), dict(x=None), dict(gamma=None),
              dict(beta=None), dict(x=ODD), dict(gamma=ODD), dict(stats=ODD), dict(ws=None), dict(ws=ODD)]
    for bad in common + [dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(eps=float("inf")), dict(y=None), dict(y=ODD)]:
        assert gn_fwd(lib, **bad) == -1, bad
    for bad in common + [dict(stats=None), dict(dy=None), dict(dgamma=None), dict(dbeta=None), dict(dx=ODD), dict(dgamma=ODD)]:
        assert gn_bwd(lib, **bad) == -1, bad
    for bad in (dict(C=16385, G=1), dict(N=(1 << 22) + 1), dict(V=1 << 37), dict(N=1 << 20, V=1 << 20)):
        assert gn_fwd(lib, **bad) == -2 and gn_bwd(lib, **bad) == -2, bad
    need = P.pyramid_group_norm_workspace_size(1, 1 << 20, 8, 4)
    assert need > 256 and gn_fwd(lib, N=1, V=1 << 20, nbytes=need - 1) == -3 and gn_bwd(lib, N=1, V=1 << 20, nbytes=need - 1) == -3
    for bad in ((0, 5, 8, 4), (2, 5, 8, 3), (2, 1 << 40, 8, 4)):
        assert P.pyramid_group_norm_workspace_size(*bad) == 0


def segment(**kw):
    f = dict(theta=0x10000, copy=0, grad=0x20000, m=0x30000, v=0x40000, mscale=0x50000, vscale=0x60000, n=10, weight_decay=0.0)
    f.update(kw)
    return P.plstm_adamw_segment(**f)


def adamw(lib, count=1, bits=32, gdtype=0, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, step=1, clock=None, lr_dev=None, scale=None, null=False, **kw):
    segs = (P.plstm_adamw_segment * 1)(segment(**kw))
    return lib.pyramid_adamw_step(count, None if null else segs, bits, gdtype, lr, b1, b2, eps, step, 0, clock, lr_dev, scale, None)


def test_adamw_refusals(lib):
    for bad in (dict(count=0), dict(count=-1), dict(null=True), dict(bits=16), dict(gdtype=2), dict(lr=-1.0), dict(lr=NAN), dict(lr=float("inf")),
                dict(b1=1.0), dict(b1=-0.1), dict(b2=NAN), dict(b2=1.5), dict(eps=0.0), dict(eps=1e-60), dict(eps=NAN), dict(step=0), dict(step=-3),
                dict(clock=ODD), dict(lr_dev=ODD), dict(scale=ODD), dict(n=-1), dict(theta=0), dict(grad=0), dict(m=0), dict(v=0),
                dict(theta=0x10001), dict(grad=0x10002), dict(copy=0x10001), dict(m=0x10002), dict(weight_decay=-0.1), dict(weight_decay=NAN),
                dict(bits=8, mscale=0), dict(bits=8, vscale=0), dict(bits=8, m=0x10004), dict(bits=8, vscale=0x10002)):
        assert adamw(lib, **bad) == -1, bad
    assert adamw(lib, n=(1 << 34) + 1) == -2
    assert adamw(lib, n=0, theta=0, grad=0, m=0, v=0) == 0        # nothing to do, nothing launched
    segs, p = (P.plstm_adamw_segment * 1)(segment()), (ctypes.c_void_p * 1)(0x70000)
    none, odd = (ctypes.c_void_p * 1)(0), (ctypes.c_void_p * 1)(0x70002)
    for m, v in ((None, p), (p, None), (none, p), (p, none), (odd, p)):
        assert lib.pyramid_adamw_moments(1, segs, m, v, None) == -1
    assert lib.pyramid_adamw_moments(0, segs, p, p, None) == -1
    assert [P.pyramid_adamw_scales(n) for n in (-1, 0, 1, 256, 257, (1 << 34) + 1)] == [0, 0, 1, 1, 2, 0]
    assert ctypes.sizeof(P.plstm_adamw_segment) == 72


def test_binding_refuses():
    x, v, w = torch.zeros((2, 4, 8)), torch.zeros(8), torch.zeros((8, 4))
    with pytest.raises(ValueError):
        P.pyramid_causal_conv_forward(x, w, v, x)
    with pytest.raises(ValueError):
        P.pyramid_selective_scan_forward(x, x, w, x, x, x)
    with pytest.raises(ValueError):
        P.pyramid_group_norm_forward(x, v, v, x, 2)
    with pytest.raises(ValueError):
        P.AdamW([v])
    with pytest.raises(ValueError):
        P.AdamW([], bits=32)
    with pytest.raises(ValueError):
        P.AdamW([v], bits=16)
    with pytest.raises(TypeError):
        P.pyramid_group_norm_forward(None, v, v, x, 2)


# ------------------------------------------------- the 64-bit forms of the GPU tests

def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def same(got, want, tol=1e-11):
    for a, b in zip(got, want):
        assert (a - b).abs().max() <= tol * (1 + b.abs().max())


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_conv_forms(act, reverse):
    B, T, I, K, lengths = 4, 9, 3, 4, [9, 0, 2, 5]
    x, w, b, state = (randn(k, *s).requires_grad_() for k, s in enumerate(((B, T, I), (I, K), (I,), (B, K - 1, I))))
    dy, dst = randn(5, B, T, I), randn(6, B, K - 1, I)
    loss, ys = 0, torch.zeros((B, T, I), dtype=torch.float64)
    for q, n in enumerate(lengths):
        seq = [state[q, k] for k in range(K - 1)] + [x[q, n - 1 - s if reverse else s] for s in range(n)]
        for s in range(n):
            a = b + sum(w[:, k] * seq[s + k] for k in range(K))
            y = a / (1 + torch.exp(-a)) if act == "silu" else a
            t = n - 1 - s if reverse else s
            ys[q, t] = y.detach()
            loss = loss + (y * dy[q, t]).sum()
        loss = loss + sum((seq[n + j] * dst[q, j]).sum() for j in range(K - 1))
    loss.backward()
    d = [t.detach() for t in (x, w, b, state)]
    (ry, _), _, kept = R.conv_forward(*d[:3], act, reverse, lengths, d[3])
    got = [v for v, _ in R.conv_backward(kept, d[1], dy, act, reverse, dst)]
    same([ry] + got, [ys, x.grad, w.grad, b.grad, state.grad])


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("gate,softplus", [(True, True), (False, False), (True, False)])
def test_selective_forms(gate, softplus, reverse):
    """Against autograd of the recurrence written step by step, and the gradient along a direction against differences."""
    B, T, I, S, lengths = 3, 11, 4, 3, [11, 0, 6]
    shapes = dict(u=(B, T, I), delta=(B, T, I), A=(I, S), Bm=(B, T, S), Cm=(B, T, S), D=(I,), z=(B, T, I), dbias=(I,), h0=(B, I, S))
    v = {k: randn(n, *s) * (0.5 if k in ("delta", "A") else 1.0) for n, (k, s) in enumerate(shapes.items())}
    dy, dhT = randn(20, B, T, I), randn(21, B, I, S)

    def loss_of(p):
        loss = 0
        for q, n in enumerate(lengths):
            h = p["h0"][q]
            for s in range(n):
                t = n - 1 - s if reverse else s
                d = p["delta"][q, t] + p["dbias"]
                d = torch.log1p(torch.exp(d)) if softplus else d
                h = torch.exp(d[:, None] * p["A"]) * h + (d * p["u"][q, t])[:, None] * p["Bm"][q, t]
                y = (h * p["Cm"][q, t]).sum(1) + p["D"] * p["u"][q, t]
                y = y * p["z"][q, t] / (1 + torch.exp(-p["z"][q, t])) if gate else y
                loss = loss + (y * dy[q, t]).sum()
            loss = loss + (h * dhT[q]).sum()
        return loss

    leaves = {k: t.clone().requires_grad_() for k, t in v.items()}
    loss_of(leaves).backward()
    ref = R.Select(v["u"], v["delta"], v["A"], v["Bm"], v["Cm"], v["D"], v["z"] if gate else None, v["dbias"], softplus, reverse,
                   lengths, v["h0"])
    got = {k: g for k, (g, _) in ref.backward(dy, dhT).items()}
    names = dict(du="u", ddelta="delta", dA="A", dB="Bm", dC="Cm", dD="D", ddelta_bias="dbias", dh0="h0", **({"dz": "z"} if gate else {}))
    assert set(names) == set(got)
    same([got[k] for k in names], [leaves[n].grad for n in names.values()])
    step = {k: randn(50 + n, *t.shape) for n, (k, t) in enumerate(v.items())}
    along = sum((got[k] * step[n]).sum() for k, n in names.items())
    e = 1e-5
    diff = (loss_of({k: t + e * step[k] for k, t in v.items()}) - loss_of({k: t - e * step[k] for k, t in v.items()})) / (2 * e)
    assert abs(float(along - diff)) <= 1e-6 * (1 + abs(float(diff)))
    same([ref.hT[1]], [v["h0"][1]])


@pytest.mark.parametrize("act", ["none", "silu"])
def test_group_norm_forms(act):
    x, w, b, dy = randn(1, 3, 4, 5, 12), randn(2, 12), randn(3, 12), randn(4, 3, 4, 5, 12)
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    y = torch.nn.functional.group_norm(leaves[0].permute(0, 3, 1, 2), 4, leaves[1], leaves[2], 1e-5).permute(0, 2, 3, 1)
    y = torch.nn.functional.silu(y) if act == "silu" else y
    y.backward(dy)
    (ry, _), _, kept = R.group_norm(x, w, b, 4, act, 1e-5)
    got = [v for v, _ in R.group_norm_backward(kept, x, w, b, dy, 4, act)]
    same([ry] + got, [y.detach()] + [t.grad for t in leaves])


def test_code_forms():
    """Values of codes are their own codes, in order; a value between two is one or the other, its mean the value."""
    for exponents, last in ((4, 120), (5, 248)):
        values = [R.code_value(k, exponents) for k in range(last + 1)]
        assert values[0] == 0 and values[-1] == 1 and all(a < b for a, b in zip(values, values[1:]))
        assert all(R.code_of(v, exponents, r) == k for k, v in enumerate(values) for r in (0, 65535))
        for k in (0, 3, 8, 50, last - 1):
            r = values[k] + (values[k + 1] - values[k]) * 0.3
            up = sum(R.code_of(r, exponents, h) == k + 1 for h in range(65536))
            assert {R.code_of(r, exponents, h) for h in (0, 65535)} == {k, k + 1} and abs(up / 65536 - 0.3) < 2.0 ** -15


def test_adamw_form():
    p, g, m, v = (randn(k, 50).float() for k in range(4))
    ours, want = p.clone(), p.clone().requires_grad_()
    opt = torch.optim.AdamW([want], lr=1e-2, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.02)
    m = v = torch.zeros(50)
    for t in range(1, 4):
        want.grad = g * t
        opt.step()
        new, _, m, v = R.adamw(ours, g * t, m, v, t, 1e-2, (0.9, 0.99), 1e-6, 0.02)
        ours = new.float()
    assert (ours - want.detach()).abs().max() <= 1e-6


def test_group_norm_of_more_groups_than_a_launch(lib):
    """A workgroup for each group: there are no more than a launch has."""
    many = dict(N=1 << 20, V=2, C=2048, G=2048)
    assert gn_fwd(lib, **many) == -2 and gn_bwd(lib, **many) == -2
    assert P.pyramid_group_norm_workspace_size(1 << 20, 2, 2048, 2048) == 0
    assert P.pyramid_group_norm_workspace_size(1 << 20, 2, 2048, 1024) > 0
