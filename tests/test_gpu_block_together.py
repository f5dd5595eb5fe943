"""Group norm, the causal convolution, the selective scan and AdamW together: a block of
them against 64-bit automatic differentiation, in captured graphs, on other streams than
the current one, two calls at once, and past 2^31 and 2^32 elements."""
from __future__ import annotations

import weakref

import pytest
import torch

import paper_1506_07452_amd as P
from paper_1506_07452_amd import network as net
from tests import block_ref as R
from tests.gpu_util import DEV, TOL, host, normwise, say
from tests.seq_ref import rounded
from tests.test_gpu_block import poisoned, sliced
from tests.test_gpu_network_norm import case
from tests.test_gpu_sequence import BF16, DTYPES, F32, Out, near, rand
from tests.test_gpu_streams import beside_busy_stream, same

pytestmark = pytest.mark.gpu

F64 = torch.float64
PROJECTED = ("w_in", "w_out")


# ------------------------------------------------------------------- the block
#
# x [N][D][H][W][C]: group norm with SiLU, one projection to u, z, delta (I channels each) and Bm, Cm
# (S states), a convolution and a selective scan along an axis, a projection back.

def block_weights(C, I, S, seed):
    w = {"gamma": rand(seed, (C,), F32, 0.2, 1.0), "beta": rand(seed + 1, (C,), F32, 0.2),
         "w_in": rand(seed + 2, (C, 3 * I + 2 * S), F32, C ** -0.5), "w_out": rand(seed + 3, (I, C), F32, I ** -0.5),
         "conv_w": rand(seed + 4, (I, 4), F32, 0.5), "conv_b": rand(seed + 5, (I,), F32, 0.2),
         "A": -torch.exp(rand(seed + 6, (I, S), F32, 0.5)), "D": rand(seed + 7, (I,), F32),
         "delta_bias": rand(seed + 8, (I,), F32, 0.5, -2.0)}
    return w


def parts_of(p, I, S):
    return torch.split(p, [I, I, I, S, S], -1)


def block_step(x, dout, w, copies, axis, reverse, groups=4, ws=None, stream=None, dtype=F32):
    """The block's output and the gradients of its weights and input by the framework's kernels."""
    I, S = w["A"].shape
    low = {k: copies[k] if dtype == BF16 else w[k] for k in ("gamma", "beta", "w_in", "w_out", "conv_w", "conv_b")}
    p = dict(conv_w=low["conv_w"], conv_b=low["conv_b"], A=w["A"], D=w["D"], delta_bias=w["delta_bias"])
    a, kept = net.group_norm_forward(x, low["gamma"], low["beta"], groups, "silu", training=True, stream=stream)
    rows = torch.matmul(a.view(-1, a.shape[-1]), low["w_in"])
    u, z, delta, Bm, Cm = parts_of(rows.view(x.shape[:-1] + (-1,)), I, S)
    y, scan = net.selective_forward(u, delta, z, Bm, Cm, p, axis, reverse, training=True, ws=ws, stream=stream)
    flat = y.view(-1, I)
    out = torch.matmul(flat, low["w_out"]).view(x.shape)
    d = dout.view(-1, x.shape[-1])
    dy = torch.matmul(d, low["w_out"].t().contiguous())
    g = net.selective_backward(dy.view(y.shape), scan, p, ws=ws, stream=stream)
    drows = torch.cat([g[k].reshape(flat.shape[0], -1) for k in ("u", "z", "delta", "Bm", "Cm")], 1)
    da = torch.matmul(drows, low["w_in"].t().contiguous())
    dx, dgamma, dbeta = net.group_norm_backward(da.view(x.shape), kept, low["gamma"], low["beta"], stream=stream)
    grads = {"gamma": dgamma, "beta": dbeta, "w_in": torch.matmul(a.view(-1, a.shape[-1]).t().float(), drows.float()),
             "w_out": torch.matmul(flat.t().float(), d.float())}
    grads.update({k: g[k] for k in ("conv_w", "conv_b", "A", "D", "delta_bias")})
    return out, dx, grads


def block64(x, w, axis, reverse, groups=4):
    """The block in 64 bits, for automatic differentiation."""
    I, S = w["A"].shape
    N, C = x.shape[0], x.shape[-1]
    xg = x.reshape(N, -1, groups, C // groups)
    mean = xg.mean((1, 3), keepdim=True)
    xh = (xg - mean) / (((xg - mean) ** 2).mean((1, 3), keepdim=True) + 1e-5).sqrt()
    a = torch.nn.functional.silu(xh.reshape(x.shape) * w["gamma"] + w["beta"])
    order = {"z": 1, "y": 2, "x": 3}

    def lines(t):
        if axis == "zyx":
            t = t.reshape(N, -1, t.shape[-1])
        else:
            t = t.movedim(order[axis], 3)
            t = t.reshape(-1, t.shape[3], t.shape[4])
        return t.flip(1) if reverse else t

    u, z, delta, Bm, Cm = (lines(t) for t in parts_of(a @ w["w_in"], I, S))
    padded = torch.cat([torch.zeros_like(u[:, :3]), u], 1)
    v = torch.nn.functional.silu(w["conv_b"] + sum(w["conv_w"][:, k] * padded[:, k:k + u.shape[1]] for k in range(4)))
    d = torch.nn.functional.softplus(delta + w["delta_bias"], threshold=1e9)
    h, ys = torch.zeros((u.shape[0], I, S), dtype=F64), []
    for t in range(u.shape[1]):
        h = torch.exp(d[:, t, :, None] * w["A"]) * h + (d[:, t] * v[:, t])[:, :, None] * Bm[:, t, None]
        ys.append(((h * Cm[:, t, None]).sum(-1) + w["D"] * v[:, t]) * torch.nn.functional.silu(z[:, t]))
    y = torch.stack(ys, 1)
    y = y.flip(1) if reverse else y
    if axis == "zyx":
        y = y.reshape(x.shape[:-1] + (I,))
    else:
        moved = x.movedim(order[axis], 3).shape[:-1] + (I,)
        y = y.reshape(moved).movedim(3, order[axis])
    return y @ w["w_out"]


@pytest.mark.parametrize("axis,reverse", [("x", False), ("y", True), ("z", False), ("zyx", True)])
def test_block_and_update(axis, reverse):
    """Output, gradients and updated weights; the gradients also against differences.  The tolerance is that of the
    network's fp32 steps."""
    C, I, S = 12, 20, 5
    shape = (2, 3, 5, 18, C)
    x, dout = rand(1, shape, F32, 1.0, 0.4), rand(2, shape, F32)
    w = block_weights(C, I, S, 10)
    say("block", axis, reverse)
    dev = {k: v.to(DEV) for k, v in w.items()}
    with torch.no_grad():
        out, dx, grads = block_step(x.to(DEV), dout.to(DEV), dev, None, axis, reverse)
    ref = {k: v.to(F64).requires_grad_() for k, v in w.items()}
    x64 = x.to(F64).requires_grad_()
    want = block64(x64, ref, axis, reverse)
    (want * dout.to(F64)).sum().backward()
    assert normwise(host(out), want.detach().numpy()) <= TOL["f32"]
    assert normwise(host(dx), x64.grad.numpy()) <= TOL["f32"]
    for k in w:
        assert normwise(host(grads[k]), ref[k].grad.numpy()) <= TOL["f32"], k
    # along a random direction of all weights, by central differences of the 64-bit form
    way = {k: rand(50 + n, v.shape, F64) for n, (k, v) in enumerate(w.items())}
    step = 1e-5
    with torch.no_grad():
        ends = [(block64(x.to(F64), {k: w[k].to(F64) + s * step * way[k] for k in w}, axis, reverse) * dout.to(F64)).sum()
                for s in (1, -1)]
    slope = float(ends[0] - ends[1]) / (2 * step)
    mine = sum(float((grads[k].cpu().double() * way[k]).sum()) for k in w)
    size = sum(float((grads[k].cpu().double() * way[k]).abs().sum()) for k in w)
    assert abs(mine - slope) <= TOL["f32"] * size
    # two updates by these gradients
    names = list(w)
    opt = P.AdamW([dev[k] for k in names], lr=1e-2, weight_decay=0.02)
    m, v = ({k: torch.zeros_like(w[k]) for k in names} for _ in range(2))
    for t in (1, 2):
        before = {k: dev[k].cpu() for k in names}
        opt.step([grads[k] for k in names])
        for k in names:
            new, bound, m[k], v[k] = R.adamw(before[k], grads[k].cpu(), m[k], v[k], t, 1e-2, (0.9, 0.999), 1e-8, 0.02)
            near(k, dev[k].cpu(), new, bound + 2.0 ** -23 * 1e-2 * 4)


@DTYPES
def test_block_inference_is_the_training_output(dtype):
    """Inference forms return the same output and keep nothing."""
    C, I, S = 16, 24, 8
    x = rand(1, (2, 4, 6, 70, C), dtype, 1.0, 0.4).to(DEV)
    w = {k: v.to(DEV) for k, v in block_weights(C, I, S, 20).items()}
    low = {k: w[k].to(dtype) for k in ("gamma", "beta", "w_in", "conv_w", "conv_b")}
    p = dict(conv_w=low["conv_w"], conv_b=low["conv_b"], A=w["A"], D=w["D"], delta_bias=w["delta_bias"])
    outs = []
    for training in (False, True):
        a, kept = net.group_norm_forward(x, low["gamma"], low["beta"], 4, "silu", training=training)
        rows = torch.matmul(a.view(-1, C), low["w_in"]).view(x.shape[:-1] + (-1,))
        u, z, delta, Bm, Cm = parts_of(rows, I, S)
        for axis in ("x", "zyx"):
            y, scan = net.selective_forward(u, delta, z, Bm, Cm, p, axis, training=training)
            assert (kept is not None) == (scan is not None) == training
            outs.append((a, y))
    same(outs[:2], outs[2:])


@DTYPES
def test_training_block_in_graphs(dtype):
    """A training step of the block with its update captured, replayed with other inputs and eager work between the
    replays, and a second graph of other weights that has the same workspace; against eager steps."""
    C, I, S = 16, 24, 8
    shape = (1, 2, 3, 400, C)
    xs = [rand(k, shape, dtype, 1.0, 0.3).to(DEV) for k in (1, 2)]
    dout = rand(3, shape, dtype).to(DEV)
    lr = torch.tensor([1e-2], device=DEV)
    scale = torch.tensor([0.5], device=DEV)
    B = shape[0] * shape[1] * shape[2]
    ws = torch.empty(max(P.pyramid_selective_scan_workspace_size(B, 400, I, S, k) for k in (0, 1)), dtype=torch.uint8, device=DEV)

    def trainer(seed, bits):
        w = {k: v.to(DEV) for k, v in block_weights(C, I, S, seed).items()}
        copies = {k: v.to(BF16) for k, v in w.items()}
        opt = P.AdamW(list(w.values()), bits=bits, copies=list(copies.values()), seed=seed, capturable=True)
        x = xs[0].clone()

        def go():
            out, dx, g = block_step(x, dout, w, copies, "x", seed == 30, ws=ws, dtype=dtype)
            opt.step([g[k] for k in w], lr=lr, grad_scale=scale)
            return out, dx, g
        return x, go, w, opt

    say("block in graphs", dtype)
    runs = []
    for captured in (False, True):
        made = [trainer(30, 32), trainer(40, 8)]
        graphs = []
        if captured:
            # what a first call sets up is done, by trainers that are not used again
            for _, go, _, _ in (trainer(30, 32), trainer(40, 8)):
                go()
            torch.cuda.synchronize()
            for x, go, w, opt in made:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    out = go()
                graphs.append((graph, out))
        seen = []
        for turn in range(4):
            for k, (x, go, w, opt) in enumerate(made):
                lr.fill_(1e-2 / (1 + turn))
                x.copy_(xs[(turn + k) % 2])
                if captured:
                    graphs[k][0].replay()
                    out = graphs[k][1]
                else:
                    out = go()
                seen.append([t.clone() for t in net._tensors((out, w, opt.moments()))])
            if captured:        # other work of the same kernels between the replays
                spare = trainer(50, 8)
                spare[1]()
                torch.cuda.synchronize()
        assert [opt.t for _, _, _, opt in made] == [4, 4]
        runs.append(seen)
    for a, b in zip(*runs):
        same(a, b)


# --------------------------------------------------------------------- streams

def entry_points(dtype):
    """name: (call(stream) on tensors made here, its outputs)."""
    def d(seed, shape, t=dtype, scale=1.0, shift=0.0):
        return rand(seed, shape, t, scale, shift).to(DEV)

    out = {}
    B, T, I, S, K = 3, 2000, 96, 16, 4
    x, dy, w, b = d(1, (B, T, I)), d(2, (B, T, I)), d(3, (I, K)), d(4, (I,))
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty((I, K), device=DEV), torch.empty(I, device=DEV)
    out["conv_forward"] = (lambda st: P.pyramid_causal_conv_forward(x, w, b, y, act="silu", stream=st), [y])
    out["conv_backward"] = (lambda st: P.pyramid_causal_conv_backward(x, w, b, dy, dx, dw, db, act="silu", stream=st), [dx, dw, db])
    delta, Bm, Cm, z = d(5, (B, T, I), scale=0.5, shift=-2.0), d(6, (B, T, S)), d(7, (B, T, S)), d(8, (B, T, I))
    A, D = -torch.exp(d(9, (I, S), F32, 0.5)), d(10, (I,), F32)
    saved = torch.empty(P.pyramid_selective_scan_saved_size(B, T, I, S), dtype=torch.uint8, device=DEV)
    P.pyramid_selective_scan_forward(x, delta, A, Bm, Cm, y, D, z, softplus=True, saved=saved)
    y2 = torch.empty_like(x)
    out["scan_forward"] = (lambda st: P.pyramid_selective_scan_forward(x, delta, A, Bm, Cm, y2, D, z, softplus=True, stream=st), [y2])
    g = [torch.empty_like(t) for t in (x, delta, A, Bm, Cm)]
    dD, dz = torch.empty_like(D), torch.empty_like(z)
    out["scan_backward"] = (lambda st: P.pyramid_selective_scan_backward(x, delta, A, Bm, Cm, saved, dy, *g, D=D, z=z, softplus=True,
                                                                         dD=dD, dz=dz, stream=st), g + [dD, dz])
    h = torch.zeros((B, I, S), device=DEV)
    y3 = torch.empty((B, 1, I), dtype=dtype, device=DEV)
    first = [t[:, :1].contiguous() for t in (x, delta, Bm, Cm, z)]
    out["scan_token"] = (lambda st: P.pyramid_selective_scan_forward(first[0], first[1], A, first[2], first[3], y3, D, first[4],
                                                                     softplus=True, hT=h, stream=st), [y3, h])
    stats, y4, dx4, dg, dB = torch.empty((B, 8, 2), device=DEV), torch.empty_like(x), torch.empty_like(x), torch.empty_like(db), \
        torch.empty_like(db)
    P.pyramid_group_norm_forward(x, b, b, y4, 8, "silu", stats)
    out["norm_forward"] = (lambda st: P.pyramid_group_norm_forward(x, b, b, y4, 8, "silu", stream=st), [y4])
    out["norm_backward"] = (lambda st: P.pyramid_group_norm_backward(x, b, b, stats, dy, dx4, dg, dB, 8, "silu", stream=st), [dx4, dg, dB])
    return out


@DTYPES
@pytest.mark.parametrize("raw", [False, True], ids=["stream", "handle"])
@pytest.mark.parametrize("name", ["conv_forward", "conv_backward", "scan_forward", "scan_backward", "scan_token", "norm_forward",
                                  "norm_backward"])
def test_call_beside_a_busy_stream(name, raw, dtype):
    call, outs = entry_points(dtype)[name]
    say("beside a busy stream", name, raw, dtype)
    call(None)
    want = [t.clone() for t in outs]
    for t in outs:
        t.fill_(float("nan"))
    torch.cuda.synchronize()
    beside_busy_stream(call, raw)
    same(outs, want)


def test_updates_and_moments_on_another_stream():
    """An update and its moments on a stream that is busy; the moments' tensors are the caller's too."""
    p, g = rand(1, (5000,), F32), rand(2, (5000,), F32).to(DEV)
    want, opts = None, []
    for _ in range(2):
        opts.append(P.AdamW([p.to(DEV)], bits=8, seed=9))
    opts[0].step([g])
    opts[0].step([g])
    want = list(net._tensors(opts[0].moments())) + opts[0].params
    say("update on another stream")

    def call(stream):
        opts[1].step([g], stream=stream)
        return opts[1].moments(stream)

    got = beside_busy_stream(call)
    torch.cuda.synchronize()
    same(list(net._tensors(got)) + opts[1].params, want)


@DTYPES
def test_two_streams_at_once(dtype):
    """Every entry point on two streams at the same time, with workspaces that the binding makes."""
    sets = [entry_points(dtype) for _ in range(2)]
    say("two streams", dtype)
    want = {}
    for name, (call, outs) in sets[0].items():
        call(None)
        want[name] = [t.clone() for t in outs]
    for s in sets:
        for _, outs in s.values():
            for t in outs:
                t.fill_(float("nan"))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for name in sets[0]:
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                s[name][0](None)
    torch.cuda.synchronize()
    for s in sets:
        for name, (_, outs) in s.items():
            same(outs, want[name])


# ------------------------------------------------------- what the binding refuses

def test_refusals():
    """Layouts, types and places that the kernels do not take."""
    B, T, I, S = 2, 6, 8, 4
    x = torch.zeros((B, T, I), device=DEV)
    w, b = torch.zeros((I, 4), device=DEV), torch.zeros(I, device=DEV)
    good = dict(x=x, w=w, bias=b, y=torch.zeros_like(x))
    P.pyramid_causal_conv_forward(**good)
    wide = torch.zeros((B, T, 2 * I), device=DEV)
    for bad in (dict(x=x.transpose(0, 1)), dict(x=x[..., ::2]), dict(x=wide[:, :, ::2]), dict(x=torch.zeros((B, T + 2, I), device=DEV)[:, 1:-1]),
                dict(x=x.double()), dict(x=x.cpu()), dict(w=w.t()), dict(w=w.to(BF16)), dict(bias=b[:4]), dict(y=wide[..., :I]),
                dict(state=torch.zeros((B, 4, I), device=DEV)), dict(lengths=torch.zeros(B, dtype=torch.int64, device=DEV)),
                dict(act="tanh"), dict(x=x[0])):
        with pytest.raises(ValueError):
            P.pyramid_causal_conv_forward(**{**good, **bad})
    A = -torch.ones((I, S), device=DEV)
    Bm = torch.zeros((B, T, S), device=DEV)
    good = dict(u=x, delta=x, A=A, Bm=Bm, Cm=Bm, y=torch.zeros_like(x))
    P.pyramid_selective_scan_forward(**good)
    for bad in (dict(A=A.to(BF16)), dict(A=A[:, :2].contiguous()), dict(Bm=Bm.to(BF16)), dict(delta=x[:, :3]), dict(z=wide[..., ::2]),
                dict(h0=torch.zeros((B, I, S), dtype=BF16, device=DEV)), dict(saved=torch.zeros(8, device=DEV)), dict(D=b.to(BF16)),
                dict(y=wide[..., :I]), dict(u=x.half()), dict(ws=torch.zeros(256, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            P.pyramid_selective_scan_forward(**{**good, **bad})
    good = dict(x=x, gamma=b, beta=b, y=torch.zeros_like(x), groups=2)
    P.pyramid_group_norm_forward(**good)
    for bad in (dict(x=wide[..., :I]), dict(gamma=b.to(BF16)), dict(stats=torch.zeros((B, 4, 2), device=DEV)), dict(y=x[:1])):
        with pytest.raises(ValueError):
            P.pyramid_group_norm_forward(**{**good, **bad})
    for bad in (dict(groups=3), dict(groups=0), dict(eps=0.0), dict(eps=float("nan")), dict(x=x[:0], y=x[:0])):
        with pytest.raises((P.PyramidLSTMError, ValueError)):
            P.pyramid_group_norm_forward(**{**good, **bad})
    p, g = [torch.zeros(10, device=DEV), torch.zeros(7, device=DEV)], [torch.ones(10, device=DEV), torch.ones(7, device=DEV)]
    for make in (lambda: P.AdamW([p[0], p[0]]), lambda: P.AdamW([p[0].to(BF16)]), lambda: P.AdamW(p, weight_decay=[0.1]), lambda: P.AdamW([]),
                 lambda: P.AdamW(p, copies=[torch.zeros(10, dtype=BF16, device=DEV)]), lambda: P.AdamW(p, bits=16),
                 lambda: P.AdamW([torch.zeros((4, 4), device=DEV).t()[1:]])):
        with pytest.raises(ValueError):
            make()
    opt = P.AdamW(p)
    for grads in (g[:1], [g[1], g[0]], [g[0], g[1].half()], [g[0], g[1].to(BF16)], [g[0], g[1].cpu()]):
        with pytest.raises(ValueError):
            opt.step(grads)
    opt.params[0].data = torch.zeros(9, device=DEV)
    with pytest.raises(ValueError):
        opt.step(g)
    assert opt.t == 0 and not opt.m[0].any()


# ------------------------------------------------------------- far and long ones

@pytest.mark.parametrize("B,T", [(9, 5), (3, 40)])
def test_wide_pitches(B, T):
    """Rows as far apart as they may be: offsets past 2^31 elements, and sequences that no wave shares."""
    I, S, K, far = 3, 4, 4, 1 << 24
    x, delta, z = rand(1, (B, T, I), BF16), rand(2, (B, T, I), BF16, 0.5, -2.0), rand(3, (B, T, I), BF16)
    Bm, Cm, dy = rand(4, (B, T, S), BF16), rand(5, (B, T, S), BF16), rand(6, (B, T, I), BF16)
    A = -torch.exp(rand(7, (I, S), F32))
    w, b = rand(8, (I, K), BF16), rand(9, (I,), BF16)
    rows = torch.empty((B, T, far), dtype=BF16, device=DEV)
    say("wide pitches", B, T)
    xd = rows[..., :I]
    zd = rows[..., far - I:]
    Bd = rows[..., 1000:1000 + S]
    for to, t in ((xd, x), (zd, z), (Bd, Bm)):
        to.copy_(t)
    y, dx, dw, db = Out((B, T, I), BF16), Out((B, T, I), BF16), Out((I, K), F32), Out((I,), F32)
    P.pyramid_causal_conv_forward(xd, w.to(DEV), b.to(DEV), y.t, act="silu")
    P.pyramid_causal_conv_backward(xd, w.to(DEV), b.to(DEV), dy.to(DEV), dx.t, dw.t, db.t, act="silu")
    (ry, by), _, kept = R.conv_forward(x, w, b, "silu", False, None, None)
    near("conv y", y.get(), ry, rounded(ry, by, BF16))
    gx, gw, gb, _ = R.conv_backward(kept, w, dy, "silu", False, None)
    near("conv dx", dx.get(), gx[0], rounded(*gx, BF16))
    near("conv dw", dw.get(), *gw)
    near("conv db", db.get(), *gb)
    ref = R.Select(x, delta, A, Bm, Cm, None, z, None, True)
    grads = ref.backward(dy)
    y, saved = Out((B, T, I), BF16), torch.empty(P.pyramid_selective_scan_saved_size(B, T, I, S), dtype=torch.uint8, device=DEV)
    how = dict(z=zd, softplus=True)
    P.pyramid_selective_scan_forward(xd, delta.to(DEV), A.to(DEV), Bd, Cm.to(DEV), y.t, saved=saved, **how)
    o = {k: Out((B, T, I), BF16) for k in ("du", "ddelta", "dz")}
    o.update(dB=Out((B, T, S), BF16), dC=Out((B, T, S), BF16), dA=Out((I, S), F32))
    P.pyramid_selective_scan_backward(xd, delta.to(DEV), A.to(DEV), Bd, Cm.to(DEV), saved, dy.to(DEV), **{k: v.t for k, v in o.items()}, **how)
    near("y", y.get(), ref.y, rounded(ref.y, ref.ey, BF16))
    for k, out in o.items():
        near(k, out.get(), grads[k][0], rounded(*grads[k], F32 if k == "dA" else BF16))


@DTYPES
def test_long_scan(dtype):
    """Many chunks of one sequence, forward and backward."""
    from tests.test_gpu_block import scan_case
    say("long scan", dtype)
    scan_case(1, 20000, 2, 2, dtype, state=True, seed=5)


@DTYPES
def test_many_channels(dtype):
    from tests.test_gpu_block import scan_case
    say("many channels", dtype)
    scan_case(1, 40, 4100, 3, dtype, state=True, seed=6)
    scan_case(2, 3, 5001, 16, dtype, seed=7, slices=True, lengths=[3, 2])


def test_padded_batch_step():
    """Single steps of a batch of which some sequences have ended: their state and output stay."""
    B, I, K, S = 4, 37, 4, 8
    lengths = torch.tensor([1, 0, 1, 0], dtype=torch.int32, device=DEV)
    for dtype in (F32, BF16):
        x, w, b = rand(1, (B, 1, I), dtype), rand(2, (I, K), dtype).to(DEV), rand(3, (I,), dtype).to(DEV)
        xd = poisoned(x, [1, 0, 1, 0])
        state = rand(4, (B, K - 1, I), dtype).to(DEV)
        old, y = state.clone(), Out((B, 1, I), dtype)
        P.pyramid_causal_conv_forward(sliced(xd), w, b, y.t, act="silu", lengths=lengths, state=state, state_out=state)
        assert torch.equal(state[1], old[1]) and torch.equal(state[3], old[3])
        assert torch.equal(state[0, -1].cpu(), x[0, 0]) and torch.equal(state[0, :-1], old[0, 1:])
        assert not y.get()[1].any() and not y.get()[3].any() and y.get()[0].isfinite().all()


GIANT = (1 << 32) + 1000


def test_giant_group_norm():
    """More than 2^32 elements: outputs at both ends and around 2^31 and 2^32, all of the sums."""
    C, G = 130, 13
    V = (GIANT + C - 1) // C
    period = 4099
    say("giant group norm")
    base = rand(1, (period, C), BF16, 1.0, 0.3).to(DEV)
    dbase = rand(2, (period, C), BF16, 0.5).to(DEV)
    x, dy, y = (torch.empty((1, V, C), dtype=BF16, device=DEV) for _ in range(3))
    whole = V // period
    for big, small in ((x, base), (dy, dbase)):
        big[0, :whole * period].view(whole, period, C).copy_(small.expand(whole, period, C))
        big[0, whole * period:] = small[:V - whole * period]
    gamma, beta = rand(3, (C,), BF16, 0.2, 1.0), rand(4, (C,), BF16, 0.2)
    stats, dg, db = torch.empty((1, G, 2), device=DEV), torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    P.pyramid_group_norm_forward(x, gamma.to(DEV), beta.to(DEV), y, G, "silu", stats)
    # the statistics of whole periods and a rest
    rest = V - whole * period
    xb = base.cpu().double()
    count = V * (C // G)
    s1 = (whole * xb.sum(0) + xb[:rest].sum(0)).view(G, -1).sum(1)
    mean = s1 / count
    dev = (xb.view(period, G, -1) - mean[:, None]) ** 2
    rstd = ((whole * dev.sum((0, 2)) + dev[:rest].sum((0, 2))) / count + 1e-5) ** -0.5
    near("mean", stats[0, :, 0].cpu(), mean, 2 * R.U * mean.abs() + 2.0 ** -48)
    near("rstd", stats[0, :, 1].cpu(), rstd, rstd * (2 * R.U + 2.0 ** -46))
    xh = ((xb.view(period, G, -1) - mean[:, None]) * rstd[:, None]).view(period, C)
    v = xh * gamma.double() + beta.double()
    ev = 8 * R.U * ((xh * gamma.double()).abs() + beta.double().abs())
    want, slope, ey, es = R.act_of(v, ev, "silu")
    places = [0, (1 << 31) // C - 2, (1 << 32) // C - 2, V - 300]
    for at in places:
        n = min(300, V - at)
        rows = [(at + k) % period for k in range(n)]
        near("y", y[0, at:at + n].cpu(), want[rows], rounded(want[rows], ey[rows], BF16))
    dx = y                      # read no more
    P.pyramid_group_norm_backward(x, gamma.to(DEV), beta.to(DEV), stats, dy, dx, dg, db, G, "silu")
    d = dbase.cpu().double()
    dv, edv = d * slope, d.abs() * (es + R.U * slope.abs())
    exh = R.U * (mean.abs() * rstd).repeat_interleave(C // G) + 5 * R.U * xh.abs()

    def over(t):
        return whole * t.sum(0) + t[:rest].sum(0)
    # a sum in fp32 within a thread's rows of a slab (at most V / 1024 of them and four waves), then in 64 bits
    chain = (V / 1024 + 64) * R.U
    near("dgamma", dg.cpu(), over(dv * xh), over(edv * xh.abs() + dv.abs() * (exh + chain * xh.abs())))
    near("dbeta", db.cpu(), over(dv), over(edv + chain * dv.abs()))
    a, ea = gamma.double() * dv, gamma.double().abs() * edv
    per = lambda t: (over(t).view(G, -1).sum(1) / count).repeat_interleave(C // G)
    m1, m2 = per(a), per(a * xh)
    em1, em2 = per(ea + chain * a.abs()), per(ea * xh.abs() + a.abs() * (exh + chain * xh.abs()))
    r = rstd.repeat_interleave(C // G)
    want = r * (a - m1 - xh * m2)
    bound = r * (ea + em1 + xh.abs() * em2 + exh * m2.abs() + 4 * R.U * (a.abs() + m1.abs() + (xh * m2).abs())) + 2 * R.U * want.abs()
    for at in places:
        n = min(300, V - at)
        rows = [(at + k) % period for k in range(n)]
        near("dx", dx[0, at:at + n].cpu(), want[rows], rounded(want[rows], bound[rows], BF16))


def test_giant_conv_and_scan():
    """More than 2^32 elements: rows at both ends of a long sequence and around 2^31 and 2^32."""
    I, K, S = 258, 4, 1
    T = (GIANT + I - 1) // I
    say("giant convolution and scan", T)
    gen = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty((1, T, I), dtype=BF16, device=DEV).normal_(generator=gen)
    w, b = rand(2, (I, K), BF16, 0.5), rand(3, (I,), BF16, 0.2)
    y = torch.empty_like(x)
    P.pyramid_causal_conv_forward(x, w.to(DEV), b.to(DEV), y, act="silu")
    places = [0, (1 << 31) // I - 100, (1 << 32) // I - 100, T - 300]

    def rows(t, at, n=300, before=0):
        return t[:, at - before:min(at + n, T)].cpu()
    for at in places:
        before = min(at, K - 1)
        part = rows(x, at, before=before)
        (ry, by), _, _ = R.conv_forward(part, w, b, "silu", False, None, None)
        near("conv y", rows(y, at), ry[:, before:], rounded(ry, by, BF16)[:, before:])
    # states fade by exp(-1) a step at least: 100 steps before a place decide it up to 2^-140 of the largest
    A = -torch.ones((I, S))
    Bm, Cm = (torch.empty((1, T, S), dtype=BF16, device=DEV).normal_(generator=gen) for _ in range(2))
    delta = torch.full((1, T, 1), 1.0, dtype=BF16, device=DEV).expand(1, T, I).contiguous()
    P.pyramid_selective_scan_forward(x, delta, A.to(DEV), Bm, Cm, y)
    for at in places:
        before = min(at, 100)
        ref = R.Select(rows(x, at, before=before), rows(delta, at, before=before), A, rows(Bm, at, before=before), rows(Cm, at, before=before))
        near("y", rows(y, at), ref.y[:, before:], rounded(ref.y, ref.ey, BF16)[:, before:] + 2.0 ** -100)


def test_giant_update():
    """A parameter of more than 2^32 elements with 8-bit moments: both ends and what lies around 2^31 and 2^32."""
    n = GIANT
    say("giant update")
    base = rand(1, (1000,), F32)
    p = torch.zeros(n, device=DEV)
    g = torch.empty(n, dtype=BF16, device=DEV)
    g.fill_(0.25)
    places = [0, (1 << 31) - 256, (1 << 32) - 256, n - n % 256 - 256]
    for at in places:
        e = min(512, n - at)
        p[at:at + e] = base[:e].to(DEV)
        g[at:at + e] = base[-e:].to(DEV)
    before = {at: (p[at:at + 512].cpu(), g[at:at + 512].cpu()) for at in places}
    opt = P.AdamW([p], lr=1e-2, bits=8, seed=77)
    opt.step([g])
    for at in places:
        p0, g0 = before[at]
        e = p0.numel()
        new, bound, m, v = R.adamw(p0, g0, torch.zeros(e), torch.zeros(e), 1, 1e-2, (0.9, 0.999), 1e-8, 0.01)
        near("p", p[at:at + e].cpu(), new, bound + 2.0 ** -23 * 1e-2 * 4)
        lo, hi = R.halves_of(e, 77, 1, 0, at)
        for x, codes, scales, half, E in ((m, opt.m[0], opt.mscale[0], lo, 4), (v, opt.v[0], opt.vscale[0], hi, 5)):
            rc, rs = R.narrow(x, E, half)
            assert torch.equal(codes[at:at + e].cpu(), rc)
            assert torch.equal(scales[at // 256:at // 256 + rs.numel()].cpu(), rs)


@pytest.mark.parametrize("reverse", [False, True])
def test_growing_states(reverse):
    """States that grow by exp(96) within a chunk, from 0 and from 1e-30: products that a chunk's growth alone would leave the
    range of."""
    B, T, I, S = 1, 192, 3, 4
    u, Bm, Cm = (rand(k, (B, T, I if k == 1 else S), F32) for k in (1, 2, 3))
    first = slice(64, None) if reverse else slice(0, 128)
    u[:, first] = 0.0                   # nothing grows but h0 and what goes back to it
    delta = torch.full((B, T, I), 0.01)
    grow = slice(128, None) if reverse else slice(0, 64)
    delta[:, grow] = 1.5
    A = torch.ones((I, S))
    h0 = torch.full((B, I, S), 1e-30)
    h0[:, 1] = 0.0
    dy = rand(4, (B, T, I), F32, 1e-30)
    ref = R.Select(u, delta, A, Bm, Cm, reverse=reverse, h0=h0)
    grads = ref.backward(dy)
    dev = [t.to(DEV) for t in (u, delta, A, Bm, Cm)]
    y, hT = Out((B, T, I), F32), Out((B, I, S), F32)
    saved = torch.empty(P.pyramid_selective_scan_saved_size(B, T, I, S), dtype=torch.uint8, device=DEV)
    say("growing states", reverse)
    P.pyramid_selective_scan_forward(*dev, y.t, reverse=reverse, h0=h0.to(DEV), hT=hT.t, saved=saved)
    o = dict(du=Out((B, T, I), F32), ddelta=Out((B, T, I), F32), dA=Out((I, S), F32), dB=Out((B, T, S), F32), dC=Out((B, T, S), F32),
             dh0=Out((B, I, S), F32))
    P.pyramid_selective_scan_backward(*dev, saved, dy.to(DEV), reverse=reverse, **{k: v.t for k, v in o.items()})
    near("y", y.get(), ref.y, rounded(ref.y, ref.ey, F32))
    near("hT", hT.get(), ref.hT, ref.ehT)
    assert ref.hT.abs().max() < 1e20 and all(torch.isfinite(v).all() for v, _ in grads.values())
    for k, out in o.items():
        near(k, out.get(), grads[k][0], rounded(*grads[k], F32))


def test_far_rows_of_long_sequences():
    """Sequences that would share waves but for the pitch of their rows, in other chunks then, with the workspace that is
    asked for: forward and backward."""
    B, T, I, S, far = 5, 44000, 3, 1, 1600
    u, delta, dy = rand(1, (B, T, I), F32), rand(2, (B, T, I), F32).abs() * 0.1, rand(3, (B, T, I), F32)
    Bm, Cm = rand(4, (B, T, S), F32), rand(5, (B, T, S), F32)
    A = -torch.exp(rand(6, (I, S), F32, 0.5))
    ref = R.Select(u, delta, A, Bm, Cm)
    grads = ref.backward(dy)
    rows = torch.empty((B, T, far), device=DEV)
    ud = rows[..., 100:100 + I]
    ud.copy_(u)
    dev = [t.to(DEV) for t in (delta, A, Bm, Cm)]
    say("far rows of long sequences")
    ws = [torch.empty(P.pyramid_selective_scan_workspace_size(B, T, I, S, k), dtype=torch.uint8, device=DEV) for k in (0, 1)]
    y, saved = Out((B, T, I), F32), torch.empty(P.pyramid_selective_scan_saved_size(B, T, I, S), dtype=torch.uint8, device=DEV)
    P.pyramid_selective_scan_forward(ud, *dev, y.t, saved=saved, ws=ws[0])
    o = dict(du=Out((B, T, I), F32), ddelta=Out((B, T, I), F32), dA=Out((I, S), F32), dB=Out((B, T, S), F32), dC=Out((B, T, S), F32))
    P.pyramid_selective_scan_backward(ud, *dev, saved, dy.to(DEV), ws=ws[1], **{k: v.t for k, v in o.items()})
    near("y", y.get(), ref.y, rounded(ref.y, ref.ey, F32))
    for k, out in o.items():
        near(k, out.get(), grads[k][0], rounded(*grads[k], F32))


@DTYPES
@pytest.mark.parametrize("axis", ["z", "y", "x", "zyx"])
def test_sweep_without_a_gate(axis, dtype):
    """A volume's selective sweep without z is the operators on its lines, forward and backward."""
    N, D, H, W, I, S = 2, 3, 4, 37, 10, 6
    u, delta = rand(1, (N, D, H, W, I), dtype).to(DEV), rand(2, (N, D, H, W, I), dtype, 0.5, -2.0).to(DEV)
    Bm, Cm = (rand(k, (N, D, H, W, S), dtype).to(DEV) for k in (3, 4))
    dy = rand(5, (N, D, H, W, I), dtype).to(DEV)
    p = dict(conv_w=rand(6, (I, 3), dtype, 0.5).to(DEV), conv_b=rand(7, (I,), dtype).to(DEV), A=-torch.exp(rand(8, (I, S), F32)).to(DEV),
             D=rand(9, (I,), F32).to(DEV), delta_bias=rand(10, (I,), F32).to(DEV))
    say("sweep without a gate", axis, dtype)
    y, kept = net.selective_forward(u, delta, None, Bm, Cm, p, axis, True, training=True)
    g = net.selective_backward(dy, kept, p)
    assert g["z"] is None
    order = {"z": (0, 2, 3, 1, 4), "y": (0, 1, 3, 2, 4), "x": (0, 1, 2, 3, 4), "zyx": (0, 1, 2, 3, 4)}[axis]
    back = [order.index(k) for k in range(5)]
    T = {"z": D, "y": H, "x": W, "zyx": D * H * W}[axis]

    def lines(t):
        return t.permute(order).reshape(-1, T, t.shape[-1]).contiguous()

    def volume(t):
        return t.view([(N, D, H, W)[k] for k in order[:4]] + [t.shape[-1]]).permute(back)

    ul, dl, Bl, Cl = (lines(t) for t in (u, delta, Bm, Cm))
    v, yl = torch.empty_like(ul), torch.empty_like(ul)
    P.pyramid_causal_conv_forward(ul, p["conv_w"], p["conv_b"], v, act="silu", reverse=True)
    saved = torch.empty(P.pyramid_selective_scan_saved_size(*ul.shape, S), dtype=torch.uint8, device=DEV)
    P.pyramid_selective_scan_forward(v, dl, p["A"], Bl, Cl, yl, p["D"], None, p["delta_bias"], True, True, saved=saved)
    assert torch.equal(volume(yl), y)
    dv, dd, dB, dC = (torch.empty_like(t) for t in (ul, dl, Bl, Cl))
    dA, dD, db = (torch.empty_like(p[k]) for k in ("A", "D", "delta_bias"))
    P.pyramid_selective_scan_backward(v, dl, p["A"], Bl, Cl, saved, lines(dy), dv, dd, dA, dB, dC, p["D"], None, p["delta_bias"], True,
                                      dD, None, db, True)
    for k, t in (("delta", dd), ("Bm", dB), ("Cm", dC)):
        assert torch.equal(volume(t), g[k]), k
    for k, t in (("A", dA), ("D", dD), ("delta_bias", db)):
        assert torch.equal(t, g[k]), k


@DTYPES
def test_large_workgroups_in_a_graph(dtype):
    """Kernels that ask for more LDS than a launch has by itself (many states, a held volume of many channels), captured
    before they have run elsewhere in other forms, replayed."""
    B, T, I, S = 2, 100, 40, 40
    u, delta, dy = rand(1, (B, T, I), dtype).to(DEV), rand(2, (B, T, I), dtype, 0.5, -2.0).to(DEV), rand(3, (B, T, I), dtype).to(DEV)
    Bm, Cm = (rand(k, (B, T, S), dtype).to(DEV) for k in (4, 5))
    A = -torch.exp(rand(6, (I, S), F32)).to(DEV)
    x, gamma = rand(7, (3, 2, 2048), dtype).to(DEV), rand(8, (2048,), dtype, 0.2, 1.0).to(DEV)

    def go():
        y, saved = torch.empty_like(u), torch.empty(P.pyramid_selective_scan_saved_size(B, T, I, S), dtype=torch.uint8, device=DEV)
        P.pyramid_selective_scan_forward(u, delta, A, Bm, Cm, y, softplus=True, saved=saved)
        g = [torch.empty_like(t) for t in (u, delta, A, Bm, Cm)]
        P.pyramid_selective_scan_backward(u, delta, A, Bm, Cm, saved, dy, *g, softplus=True)
        z, stats, dx = torch.empty_like(x), torch.empty((3, 16, 2), device=DEV), torch.empty_like(x)
        dg, db = torch.empty(2048, device=DEV), torch.empty(2048, device=DEV)
        P.pyramid_group_norm_forward(x, gamma, gamma, z, 16, "silu", stats)
        P.pyramid_group_norm_backward(x, gamma, gamma, stats, z, dx, dg, db, 16, "silu")
        return [y] + g + [z, dx, dg, db]

    say("large workgroups in a graph", dtype)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = go()
    for _ in range(3):
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        want = go()
        torch.cuda.synchronize()
        same(got, want)


@pytest.mark.parametrize("bits", [32, 8])
def test_network_updates(bits):
    """A normed network's parameters and gradients through AdamW, decay for the weights only."""
    d, _ = case([16, 32], True, 61, (1, 0))
    params = net.network_parameters(d["layers"], d["fcs"], d["head"], d["norms"])
    decay = [0.05 if p.dim() > 1 else 0.0 for p in params]
    opt = P.AdamW(params, lr=1e-3, weight_decay=decay, bits=bits, seed=4)
    m, v = ([torch.zeros(p.shape) for p in params] for _ in range(2))
    say("network updates", bits)
    for t in (1, 2):
        grads = net.network_gradients(net.network_train_step(d["x"], d["layers"], d["fcs"], d["head"], d["labels"], norms=d["norms"]))
        before = [p.cpu() for p in params]
        opt.step(grads)
        for k, (p, g) in enumerate(zip(params, grads)):
            new, bound, m[k], v[k] = R.adamw(before[k], g.cpu(), m[k], v[k], t, 1e-3, (0.9, 0.999), 1e-8, decay[k])
            near("p", p.cpu(), new, bound + 2.0 ** -23 * 1e-3 * 4)
        if bits == 8:
            m, v = ([x[j].cpu() for x in opt.moments()] for j in (0, 1))
        else:
            assert all(torch.equal(a.cpu(), b) for a, b in zip(opt.m + opt.v, m + v))


@pytest.mark.parametrize("name", ["conv_backward", "scan_forward", "scan_backward", "norm_forward", "norm_backward"])
def test_workspace_lives_through_the_call(name, monkeypatch):
    """A workspace that the binding makes is not given back before its call has been made."""
    call, _ = entry_points(F32)[name]
    made, seen, run = [], [], P._run
    temporary = P._temporary

    def tracked(*args):
        ws = temporary(*args)
        made.append(weakref.ref(ws))
        return ws

    def watched(*args):
        seen.extend(ref() is not None for ref in made)
        run(*args)

    monkeypatch.setattr(P, "_temporary", tracked)
    monkeypatch.setattr(P, "_run", watched)
    say("workspace through the call", name)
    call(None)
    torch.cuda.synchronize()
    assert seen == [True]


@DTYPES
@pytest.mark.parametrize("T", [2, 5, 100, 700])
def test_conv_state_in_place_of_runs(T, dtype):
    """The state after in the place of the one before, where a sequence has several runs and where it is shorter than the taps."""
    B, I, K = 3, 21, 8
    x, w, b = rand(1, (B, T, I), dtype).to(DEV), rand(2, (I, K), dtype, 0.5).to(DEV), rand(3, (I,), dtype).to(DEV)
    lengths = torch.tensor([T, 0, T // 2], dtype=torch.int32, device=DEV)
    before = rand(4, (B, K - 1, I), dtype).to(DEV)
    after, y, there = torch.empty_like(before), torch.empty_like(x), torch.empty_like(x)
    say("convolution's state in place", T, dtype)
    for reverse in (False, True):
        how = dict(act="silu", reverse=reverse, lengths=lengths)
        P.pyramid_causal_conv_forward(x, w, b, y, state=before, state_out=after, **how)
        state = before.clone()
        P.pyramid_causal_conv_forward(x, w, b, there, state=state, state_out=state, **how)
        assert torch.equal(there, y) and torch.equal(state, after)


def test_counted_updates_without_gradients():
    """A counted update of tensors of which some, or all, have no gradient: the count goes on, those tensors stay."""
    p = [rand(k, (300,), F32).to(DEV) for k in (1, 2)]
    g = rand(3, (300,), F32).to(DEV)
    kept = [t.clone() for t in p]
    opt = P.AdamW(p, lr=1e-2, capturable=True)
    opt.step([None, None])
    opt.step([None, g])
    say("counted updates")
    assert opt.t == 2 and torch.equal(p[0], kept[0])
    new, bound, m, v = R.adamw(kept[1].cpu(), g.cpu(), torch.zeros(300), torch.zeros(300), 2, 1e-2, (0.9, 0.999), 1e-8, 0.01)
    near("p", p[1].cpu(), new, bound + 2.0 ** -23 * 1e-2 * 4)
    assert torch.equal(opt.m[1].cpu(), m) and torch.equal(opt.v[1].cpu(), v) and not opt.m[0].any()
