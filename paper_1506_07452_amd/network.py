"""Stacked PyraMiD-LSTM networks on the GPU, composed from the C entry points.

Fig. 3 / Section 2.3: PyraMiD-LSTM layer -> per-voxel FC + tanh, repeated;
the last FC layer feeds a per-voxel softmax.  This module only allocates
tensors with torch and calls the library (every arithmetic step runs in the
HIP kernels); gradients flow through the same entry points in reverse.
Beyond Fig. 3 a layer's output may be normed over its channels before its FC
(`norms`), and a training step may hold what the layers keep for their
backward in 8 bits (`checkpoint8`).
Group norm and selective sweeps along the lines of a volume, the blocks of state
space models over volumes, stand beside them.
"""
from __future__ import annotations

import functools
import inspect
from dataclasses import dataclass
from typing import List, Optional, Tuple

import torch

from . import (_torch_stream, checkpoint8_empty, plstm_shape, pyramid_checkpoint8_pack,
               pyramid_causal_conv_backward, pyramid_causal_conv_forward,
               pyramid_checkpoint8_unpack, pyramid_fc_tanh_backward, pyramid_fc_tanh_forward,
               pyramid_group_norm_backward, pyramid_group_norm_forward,
               pyramid_head_forward, pyramid_head_forward_supported,
               pyramid_head_train, pyramid_head_workspace_size, pyramid_layer_norm_backward,
               pyramid_layer_norm_forward, pyramid_lstm_backward,
               pyramid_lstm_forward, pyramid_lstm_saved_size, pyramid_lstm_workspace_size,
               pyramid_lstm2d_backward, pyramid_lstm2d_forward, pyramid_lstm2d_saved_size,
               pyramid_scan_backward, pyramid_scan_forward, pyramid_scan_saved_size,
               pyramid_selective_scan_backward, pyramid_selective_scan_forward,
               pyramid_selective_scan_saved_size, pyramid_softmax_ce, shape2d_for, shape_for)


@dataclass
class LayerW:
    wx: torch.Tensor      # [6][4O][C][K][K]
    wh: torch.Tensor      # [6][4O][O][K][K]
    b: torch.Tensor       # [6][4O]

    @property
    def O(self):
        return self.wh.shape[2]

    @property
    def K(self):
        return self.wh.shape[-1]


def layer_forward(x: torch.Tensor, L: LayerW, training: bool = False, ws=None, stream=None):
    """One layer; returns (h, saved or None)."""
    s = shape_for(x, L.O, L.K)
    h = torch.empty(x.shape[:-1] + (L.O,), dtype=x.dtype, device=x.device)
    saved = None
    if training:
        saved = torch.empty(pyramid_lstm_saved_size(s), dtype=torch.uint8, device=x.device)
    pyramid_lstm_forward(s, x, L.wx, L.wh, L.b, h, saved, ws, stream)
    return h, saved


def layer_backward(x, L: LayerW, saved, dh, want_dx=True, ws=None, stream=None):
    s = shape_for(x, L.O, L.K)
    dx = torch.empty_like(x) if want_dx else None
    dwx, dwh, db = (torch.empty_like(t, dtype=torch.float32) for t in (L.wx, L.wh, L.b))
    pyramid_lstm_backward(s, x, L.wx, L.wh, L.b, saved, dh, dx, dwx, dwh, db, ws, stream)
    return dx, dwx, dwh, db


def layer2d_forward(x: torch.Tensor, L: LayerW, training: bool = False, ws=None, stream=None):
    """2D layer over x [N][H][W][C] (weights [4][4O][C|O][K], b [4][4O]);
    returns (h, saved or None)."""
    s = shape2d_for(x, L.O, L.K)
    h = torch.empty(x.shape[:-1] + (L.O,), dtype=x.dtype, device=x.device)
    saved = None
    if training:
        saved = torch.empty(pyramid_lstm2d_saved_size(s), dtype=torch.uint8, device=x.device)
    pyramid_lstm2d_forward(s, x, L.wx, L.wh, L.b, h, saved, ws, stream)
    return h, saved


def layer2d_backward(x, L: LayerW, saved, dh, want_dx=True, ws=None, stream=None):
    s = shape2d_for(x, L.O, L.K)
    dx = torch.empty_like(x) if want_dx else None
    dwx, dwh, db = (torch.empty_like(t, dtype=torch.float32) for t in (L.wx, L.wh, L.b))
    pyramid_lstm2d_backward(s, x, L.wx, L.wh, L.b, saved, dh, dx, dwx, dwh, db, ws, stream)
    return dx, dwx, dwh, db


def norm_forward(h: torch.Tensor, gamma, beta, eps: float = 1e-5, training: bool = False,
                 checkpoint8: bool = False, stream=None):
    """Layer norm over the last axis of h; returns (y, kept): kept is None for
    inference, else what norm_backward needs, with h itself or (checkpoint8)
    its 8-bit checkpoint."""
    C = h.shape[-1]
    rows = h.view(-1, C)
    y = torch.empty_like(h)
    if not training:
        pyramid_layer_norm_forward(rows, gamma, beta, y.view(-1, C), eps=eps, stream=stream)
        return y, None
    stats = torch.empty((rows.shape[0], 2), dtype=torch.float32, device=h.device)
    q, scale = checkpoint8_empty(rows) if checkpoint8 else (None, None)
    pyramid_layer_norm_forward(rows, gamma, beta, y.view(-1, C), stats, q, scale, eps=eps,
                               stream=stream)
    return y, (rows if q is None else q, scale, stats)


def norm_backward(kept, gamma, dy, want_dx=True, ws=None, stream=None):
    """(dx or None, dgamma, dbeta) of norm_forward for dy of its output's shape."""
    x, scale, stats = kept
    rows = dy.view(x.shape)
    dx = torch.empty_like(rows) if want_dx else None
    dgamma, dbeta = (torch.empty(x.shape[1], dtype=torch.float32, device=dy.device)
                     for _ in range(2))
    pyramid_layer_norm_backward(x, gamma, stats, rows, dx, dgamma, dbeta, xscale=scale, ws=ws,
                                stream=stream)
    return None if dx is None else dx.view(dy.shape), dgamma, dbeta


def _sequences(x, axis):
    """The [B][T][I] view of a volume [N][D][H][W][C] whose middle axis is `axis`."""
    if x.dim() != 5 or axis not in ("z", "y", "x"):
        raise ValueError("x must be [N][D][H][W][C] and axis one of z, y, x")
    N, D, H, W, C = x.shape
    return x.view({"z": (N, D, H * W * C), "y": (N * D, H, W * C), "x": (N * D * H, W, C)}[axis])


def scan_forward(g: torch.Tensor, u: torch.Tensor, axis: str, reverse: bool = False,
                 training: bool = False, ws=None, stream=None):
    """Linear sweep of a volume along `axis` ("z", "y" or "x"; from the far side
    with `reverse`), gates g and inputs u [N][D][H][W][C]; returns (h, saved or
    None)."""
    gs, us = _sequences(g, axis), _sequences(u, axis)
    h = torch.empty_like(g)
    saved = None
    if training:
        saved = torch.empty(pyramid_scan_saved_size(*gs.shape), dtype=torch.uint8, device=g.device)
    pyramid_scan_forward(gs, us, _sequences(h, axis), reverse, saved=saved, ws=ws, stream=stream)
    return h, saved


def scan_backward(g, u, saved, dh, axis: str, reverse: bool = False, ws=None, stream=None):
    """(dg, du) of scan_forward; g and u are its inputs, or (codes, scale) pairs of
    their 8-bit checkpoints."""
    (g, gscale), (u, uscale) = (t if isinstance(t, tuple) else (t, None) for t in (g, u))
    dg, du = torch.empty_like(dh), torch.empty_like(dh)
    pyramid_scan_backward(_sequences(g, axis), _sequences(u, axis), saved, _sequences(dh, axis),
                          _sequences(dg, axis), _sequences(du, axis), reverse, gscale=gscale,
                          uscale=uscale, ws=ws, stream=stream)
    return dg, du


def _saved_arrays(saved, s: plstm_shape):
    """The fp32 arrays (gates, c^d, h^d) of a training forward's saved buffer:
    each starts at the next 256-byte boundary."""
    cells = 6 * s.N * s.D * s.H * s.W * s.O
    out, off = [], 0
    for n in (4 * cells, cells, cells):
        off = -(-off // 256) * 256
        out.append(saved[off:off + 4 * n].view(torch.float32))
        off += 4 * n
    if not saved.numel() == off == pyramid_lstm_saved_size(s):
        raise ValueError("saved has %d bytes, its arrays %d and a buffer of this shape %d" % (
            saved.numel(), off, pyramid_lstm_saved_size(s)))
    return out


def saved_pack(saved, s: plstm_shape, stream=None):
    """8-bit checkpoints of a saved buffer's arrays (about a quarter of its bytes)."""
    out = []
    for a in _saved_arrays(saved, s):
        q, scale = checkpoint8_empty(a)
        pyramid_checkpoint8_pack(a, q, scale, stream)
        out.append((q, scale))
    return out


def saved_unpack(packed, s: plstm_shape, stream=None):
    """A saved buffer with the values of saved_pack's checkpoints."""
    saved = torch.empty(pyramid_lstm_saved_size(s), dtype=torch.uint8, device=packed[0][0].device)
    for (q, scale), a in zip(packed, _saved_arrays(saved, s)):
        pyramid_checkpoint8_unpack(q, scale, a, stream)
    return saved


def workspace_for(x_shape, hidden: List[int], fc: bool, dtype, training: bool, device):
    """One workspace big enough for every layer of a network whose FC layers
    are twice as wide as the layer before (3 x 3 filters)."""
    shapes, C = [], x_shape[-1]
    for O in hidden:
        shapes.append((C, O, 3))
        C = 2 * O if fc else O
    return workspace_for_layers(x_shape, shapes, dtype, training, device)


def workspace_for_layers(x_shape, shapes, dtype, training: bool, device):
    """One workspace big enough for layers of (input channels, hidden units,
    filter size) `shapes` over the volume of `x_shape`."""
    need = 256
    for C, O, K in shapes:
        s = plstm_shape(*x_shape[:-1], C, O, 0 if dtype == torch.float32 else 1, K)
        need = max(need, pyramid_lstm_workspace_size(s, int(training)))
    return torch.empty(need, dtype=torch.uint8, device=device)


def _tensors(out):
    """The tensors in a result, however deep."""
    if isinstance(out, torch.Tensor):
        yield out
    elif isinstance(out, (dict, list, tuple)):
        for v in out.values() if isinstance(out, dict) else out:
            yield from _tensors(v)


def _on_its_stream(fn):
    """A network call given `stream` takes all its memory from that stream: what it
    drops on its way or when it returns goes to later work of that stream alone,
    never to tensors that another stream may write while the call's work has yet to
    read them.  What it returns is the caller's current stream's as well."""
    at = list(inspect.signature(fn).parameters).index("stream")

    @functools.wraps(fn)
    def call(x, *args, **kw):
        stream = args[at - 1] if len(args) >= at else kw.get("stream")
        if stream is None:
            return fn(x, *args, **kw)
        caller = torch.cuda.current_stream(x.device)
        with torch.cuda.stream(_torch_stream(stream, x.device)):
            out = fn(x, *args, **kw)
        for t in _tensors(out):
            t.record_stream(caller)
        return out
    return call


def _lines(x, axis):
    """[lines][T][n]: a volume's [N][D][H][W][n] lines along `axis` ("zyx": all its voxels in
    raster order); a copy for "z" and "y"."""
    if x is None:
        return None
    if x.dim() != 5 or axis not in ("z", "y", "x", "zyx"):
        raise ValueError("x must be [N][D][H][W][C] and axis one of z, y, x, zyx")
    if axis == "zyx":
        return x.reshape(x.shape[0], -1, x.shape[-1])
    if axis != "x":
        x = x.movedim({"z": 1, "y": 2}[axis], 3).contiguous()
    return x.reshape(-1, x.shape[3], x.shape[4])


def _unlines(t, shape, axis):
    """The volume [N][D][H][W][n] of _lines' output for a volume of `shape`."""
    if t is None:
        return None
    N, D, H, W = shape[:4]
    if axis == "z":
        return t.view(N, H, W, D, -1).movedim(3, 1).contiguous()
    if axis == "y":
        return t.view(N, D, W, H, -1).movedim(3, 2).contiguous()
    return t.view(N, D, H, W, -1)


@_on_its_stream
def group_norm_forward(x, gamma, beta, groups: int, act: str = "none", eps: float = 1e-5,
                       training: bool = False, ws=None, stream=None):
    """Group norm over the voxels of each volume x [N][...][C] with an activation ("none" or
    "silu"); returns (y, kept): kept is None for inference, else what
    group_norm_backward needs."""
    y = torch.empty_like(x)
    stats = None
    if training:
        stats = torch.empty((x.shape[0], groups, 2), dtype=torch.float32, device=x.device)
    pyramid_group_norm_forward(x, gamma, beta, y, groups, act, stats, eps, ws, stream)
    return y, (x, stats, groups, act) if training else None


@_on_its_stream
def group_norm_backward(dy, kept, gamma, beta, want_dx: bool = True, ws=None, stream=None):
    """(dx or None, dgamma, dbeta) of group_norm_forward."""
    x, stats, groups, act = kept
    dx = torch.empty_like(x) if want_dx else None
    dgamma, dbeta = (torch.empty(x.shape[-1], dtype=torch.float32, device=x.device) for _ in range(2))
    pyramid_group_norm_backward(x, gamma, beta, stats, dy, dx, dgamma, dbeta, groups, act, ws, stream)
    return dx, dgamma, dbeta


@_on_its_stream
def selective_forward(u, delta, z, Bm, Cm, p, axis: str, reverse: bool = False, training: bool = False,
                      ws=None, stream=None):
    """Selective sweep of a volume: a causal convolution with SiLU of u, then a selective scan of it gated
    by z (or None), along the lines of `axis` ("z", "y" or "x", "zyx": all voxels in raster order;
    from the far side with `reverse`).  u, delta, z [N][D][H][W][I], Bm, Cm [N][D][H][W][S]; p: a dict
    of conv_w [I][K], conv_b [I] in their dtype and A [I][S], D, delta_bias [I] fp32 (conv_b, D and
    delta_bias may be None: zeros).
    Returns (y, kept): kept is None for inference, else what selective_backward needs."""
    shape = u.shape
    u, delta, z, Bm, Cm = (_lines(t, axis) for t in (u, delta, z, Bm, Cm))
    v, y = torch.empty_like(u), torch.empty_like(u)
    pyramid_causal_conv_forward(u, p["conv_w"], p["conv_b"], v, act="silu", reverse=reverse, stream=stream)
    saved = None
    if training:
        saved = torch.empty(pyramid_selective_scan_saved_size(*u.shape, p["A"].shape[1]), dtype=torch.uint8,
                            device=u.device)
    pyramid_selective_scan_forward(v, delta, p["A"], Bm, Cm, y, p["D"], z, p["delta_bias"], True, reverse,
                                   saved=saved, ws=ws, stream=stream)
    return _unlines(y, shape, axis), (u, v, delta, z, Bm, Cm, saved, axis, reverse) if training else None


@_on_its_stream
def selective_backward(dy, kept, p, ws=None, stream=None):
    """Gradients of selective_forward: a dict of u, delta, z, Bm, Cm (volumes) and conv_w, conv_b,
    A, D, delta_bias (fp32); None for what was None."""
    u, v, delta, z, Bm, Cm, saved, axis, reverse = kept
    shape, dy = dy.shape, _lines(dy, axis)
    g = {k: None if t is None else torch.empty_like(t)
         for k, t in (("v", v), ("delta", delta), ("z", z), ("Bm", Bm), ("Cm", Cm), ("u", u))}
    for k in ("conv_w", "conv_b", "A", "D", "delta_bias"):
        g[k] = None if p[k] is None else torch.empty_like(p[k], dtype=torch.float32)
    pyramid_selective_scan_backward(v, delta, p["A"], Bm, Cm, saved, dy, g["v"], g["delta"], g["A"], g["Bm"],
                                    g["Cm"], p["D"], z, p["delta_bias"], True, g["D"], g["z"], g["delta_bias"],
                                    reverse, ws=ws, stream=stream)
    pyramid_causal_conv_backward(u, p["conv_w"], p["conv_b"], g.pop("v"), g["u"], g["conv_w"], g["conv_b"],
                                 act="silu", reverse=reverse, stream=stream)
    for k in ("u", "delta", "z", "Bm", "Cm"):
        g[k] = _unlines(g[k], shape, axis)
    return g


@_on_its_stream
def network_forward(x, layers: List[LayerW], fcs: List[Tuple[torch.Tensor, torch.Tensor]],
                    head: Tuple[torch.Tensor, torch.Tensor], labels: Optional[torch.Tensor] = None,
                    training: bool = False, ws=None, stream=None, loss: str = "ce", norms=None,
                    checkpoint8: bool = False):
    """Returns dict: 'p' [M][K] fp32, 'loss' (device scalar, with labels),
    'acts' (per-layer inputs/outputs and saved activations for training).
    loss: "ce" (mean cross-entropy) or "sq" (squared error, Eq. (14)).
    norms: per layer None or (gamma, beta) [O], a layer norm of its output over
    the channels before its FC.  checkpoint8 (training): as in
    network_train_step."""
    N, D, H, W, _ = x.shape
    M = N * D * H * W
    if len(fcs) not in (len(layers), len(layers) - 1):
        raise ValueError("one hidden FC layer per PyraMiD-LSTM layer, or none after the last")
    K = head[0].shape[0]
    # inference with bf16 storage: the last FC and the softmax as one pass
    # (the last layer's act then has no "y")
    fused = (labels is None and not training and len(fcs) == len(layers) and
             x.dtype == torch.bfloat16 and
             pyramid_head_forward_supported(x.dtype, layers[-1].O, fcs[-1][0].shape[0], K))
    a = x
    acts = []
    for li, L in enumerate(layers):
        act = _layer_act(a, li, layers, norms, training, checkpoint8, ws, stream)
        h = a = act["h"]
        if fused and li == len(layers) - 1:
            acts.append(act)
            p = torch.empty((M, K), dtype=torch.float32, device=x.device)
            pyramid_head_forward(h.view(M, -1), fcs[li][0], fcs[li][1], head[0], head[1], p,
                                 stream)
            return {"p": p, "acts": acts}
        if li < len(fcs):
            wf, bf = fcs[li]
            y = torch.empty((N, D, H, W, wf.shape[0]), dtype=a.dtype, device=a.device)
            pyramid_fc_tanh_forward(h.view(M, -1), wf, bf, y.view(M, -1), stream)
            act["y"] = y
            a = y
        acts.append(act)
    p = torch.empty((M, K), dtype=torch.float32, device=x.device)
    out = {"p": p, "acts": acts}
    if labels is None:
        pyramid_softmax_ce(a.view(M, -1), head[0], head[1], p, stream=stream)
        return out
    if loss not in ("ce", "sq"):
        raise ValueError("loss must be 'ce' or 'sq'")
    lval = torch.empty(1, dtype=torch.float32, device=x.device)
    out["loss"] = lval
    if training:
        dlast = torch.empty((M, a.shape[-1]), dtype=torch.float32, device=x.device)
        dw = torch.empty_like(head[0])
        db = torch.empty_like(head[1])
        pyramid_softmax_ce(a.view(M, -1), head[0], head[1], p, labels, lval, dlast, dw, db,
                           stream=stream, squared=loss == "sq")
        out.update({"dlast": dlast, "head_grad": (dw, db)})
    else:
        pyramid_softmax_ce(a.view(M, -1), head[0], head[1], p, labels, lval, stream=stream,
                           squared=loss == "sq")
    return out


def _layer_act(a, li, layers, norms, training, checkpoint8, ws, stream):
    """Layer li and its norm on input a (norms: one entry per layer): 'h' is what the FC reads; for training
    'saved' and, with a norm, 'kept'.  With checkpoint8 a layer below the last
    one keeps its saved buffer, and its norm's input, in 8 bits ('packed'): until
    its backward they lie idle."""
    if norms is not None and len(norms) != len(layers):
        raise ValueError("norms must have an entry (gamma, beta) or None per layer")
    L = layers[li]
    eight = training and checkpoint8 and li < len(layers) - 1
    h, saved = layer_forward(a, L, training, ws, stream)
    act = {"in": a, "h": h, "saved": saved}
    if eight:
        act["packed"] = saved_pack(saved, shape_for(a, L.O, L.K), stream)
        act["saved"] = None
    if norms is not None and norms[li] is not None:
        act["h"], act["kept"] = norm_forward(h, *norms[li], training=training, checkpoint8=eight,
                                             stream=stream)
    return act


def _layer_act_backward(act, li, layers, norms, dh, ws, stream):
    """(dx or None, (dwx, dwh, db), (dgamma, dbeta) or None) from the gradient of
    act's 'h'."""
    L, dn = layers[li], None
    if "kept" in act:
        dh, dgamma, dbeta = norm_backward(act["kept"], norms[li][0], dh, stream=stream)
        dn = (dgamma, dbeta)
    saved = act["saved"]
    if "packed" in act:
        saved = saved_unpack(act.pop("packed"), shape_for(act["in"], L.O, L.K), stream)
    dx, dwx, dwh, db = layer_backward(act["in"], L, saved, dh.view(act["h"].shape),
                                      want_dx=li > 0, ws=ws, stream=stream)
    return dx, (dwx, dwh, db), dn


@_on_its_stream
def network_train_step(x, layers, fcs, head, labels, ws=None, stream=None, fused_head=True,
                       loss="ce", norms=None, checkpoint8=False):
    """Forward + back-propagation through the whole network (fp32).
    Returns dict with 'loss', 'p', 'head' (dw, db), 'fcs' [(dw, db)],
    'layers' [(dwx, dwh, db)] and, with norms (see network_forward), 'norms'
    [(dgamma, dbeta) or None].  checkpoint8: the layers below the last hold their saved
    buffers, and the inputs of their norms, in 8 bits until their backward
    (gradients are then those of activations rounded to a 127th of the largest
    of 64).  With `fused_head` (default) the last FC + tanh,
    the softmax head, the loss and their backward run as one pass over the
    voxels (pyramid_head_train) where it covers the widths."""
    N, D, H, W, _ = x.shape
    M = N * D * H * W
    nl = len(layers)
    O_last, F_last, K = layers[-1].O, fcs[-1][0].shape[0], head[0].shape[0]
    if not (fused_head and loss == "ce" and len(fcs) == nl and
            pyramid_head_workspace_size(M, O_last, F_last, K) > 0):
        return _train_step_unfused(x, layers, fcs, head, labels, ws, stream, loss, norms,
                                   checkpoint8)
    a = x
    acts = []
    for li in range(nl):
        act = _layer_act(a, li, layers, norms, True, checkpoint8, ws, stream)
        h = act["h"]
        if li < nl - 1:
            wf, bf = fcs[li]
            y = torch.empty((N, D, H, W, wf.shape[0]), dtype=a.dtype, device=a.device)
            pyramid_fc_tanh_forward(h.view(M, -1), wf, bf, y.view(M, -1), stream)
            act["y"] = y
            a = y
        acts.append(act)
    p = torch.empty((M, K), dtype=torch.float32, device=x.device)
    lval = torch.empty(1, dtype=torch.float32, device=x.device)
    dh = torch.empty((M, O_last), dtype=torch.float32, device=x.device)
    wf, bf = fcs[-1]
    dwf, dbf = torch.empty_like(wf), torch.empty_like(bf)
    dw, db = torch.empty_like(head[0]), torch.empty_like(head[1])
    pyramid_head_train(acts[-1]["h"].view(M, O_last), wf, bf, head[0], head[1], labels, p, lval,
                       dh, dwf, dbf, dw, db, stream=stream)
    fc_grads = [None] * len(fcs)
    layer_grads, norm_grads = [None] * nl, [None] * nl
    fc_grads[-1] = (dwf, dbf)
    g = None
    for li in range(nl - 1, -1, -1):
        act = acts[li]
        O = act["h"].shape[-1]
        if li < nl - 1:
            wf, _ = fcs[li]
            dh = torch.empty((M, O), dtype=torch.float32, device=x.device)
            dwf, dbf = torch.empty_like(wf), torch.empty(wf.shape[0], device=x.device)
            pyramid_fc_tanh_backward(act["h"].view(M, O), wf, act["y"].view(M, -1),
                                     g.view(M, -1), dh, dwf, dbf, stream=stream)
            fc_grads[li] = (dwf, dbf)
        g, layer_grads[li], norm_grads[li] = _layer_act_backward(act, li, layers, norms, dh, ws,
                                                                 stream)
        act = acts[li] = None       # before the next layer's buffers are there
    out = {"loss": lval, "p": p, "head": (dw, db), "fcs": fc_grads, "layers": layer_grads}
    if norms is not None:
        out["norms"] = norm_grads
    return out


def _train_step_unfused(x, layers, fcs, head, labels, ws=None, stream=None, loss="ce", norms=None,
                        checkpoint8=False):
    """network_train_step composed from the separate FC / softmax entry points."""
    out = network_forward(x, layers, fcs, head, labels, training=True, ws=ws, stream=stream,
                          loss=loss, norms=norms, checkpoint8=checkpoint8)
    acts = out["acts"]
    g = out["dlast"]
    N, D, H, W, _ = x.shape
    M = N * D * H * W
    fc_grads = [None] * len(fcs)
    layer_grads, norm_grads = [None] * len(layers), [None] * len(layers)
    for li in range(len(layers) - 1, -1, -1):
        act = acts[li]
        O = act["h"].shape[-1]
        if li < len(fcs):
            wf, _ = fcs[li]
            dh = torch.empty((M, O), dtype=torch.float32, device=x.device)
            dwf, dbf = torch.empty_like(wf), torch.empty(wf.shape[0], device=x.device)
            pyramid_fc_tanh_backward(act["h"].view(M, O), wf, act["y"].view(M, -1),
                                     g.view(M, -1), dh, dwf, dbf, stream=stream)
            fc_grads[li] = (dwf, dbf)
        else:
            dh = g      # the output layer reads h directly
        dx, layer_grads[li], norm_grads[li] = _layer_act_backward(act, li, layers, norms, dh, ws,
                                                                  stream)
        act = acts[li] = None       # before the next layer's buffers are there
        if li > 0:
            g = dx
    res = {"loss": out["loss"], "p": out["p"], "head": out["head_grad"], "fcs": fc_grads,
           "layers": layer_grads}
    if norms is not None:
        res["norms"] = norm_grads
    return res


def network_parameters(layers, fcs, head, norms=None):
    """Every parameter tensor of a network, for RMSprop or AdamW, in the order of
    `network_gradients`: per layer (wx, wh, b), per hidden FC (w, b), head, per
    norm (gamma, beta)."""
    out = []
    for L in layers:
        out += [L.wx, L.wh, L.b]
    for w, b in fcs:
        out += [w, b]
    out += [head[0], head[1]]
    for n in norms or []:
        out += list(n or ())
    return out


def network_gradients(g):
    """The gradients of a `network_train_step` result, in the order of
    `network_parameters`."""
    out = []
    for t in g["layers"]:
        out += list(t)
    for t in g["fcs"]:
        out += list(t)
    out += [g["head"][0], g["head"][1]]
    for n in g.get("norms", []):
        out += list(n or ())
    return out


def grid_axis(extent, size, stride):
    """Tile origins along one axis of `extent` voxels for tiles of `size`
    (cut to the extent) advancing by `stride`: n = ceil((extent - size) /
    stride) + 1 tiles, the i-th at min(i * stride, extent - size), so the
    last one ends flush with the axis.  Returns (origins, size)."""
    if extent < 1 or size < 1 or stride < 1:
        raise ValueError("extent, tile size and stride must be positive")
    size = min(size, extent)
    span = extent - size
    n = -(-span // stride) + 1
    return [min(i * stride, span) for i in range(n)], size


@_on_its_stream
def network_infer_volume(x, layers, fcs, head, tile, stride=None, sigma_scale=0.25, ws=None,
                         stream=None, origins=None, norms=None):
    """Class probabilities [N][D][H][W][K] of a volume processed as sub-volumes
    (Section 3, "Sub-volumes and Augmentation"): tiles of size `tile` (d, h, w),
    each run through the network on its own and stitched with Gaussian weights
    (sigma = sigma_scale x tile extent).  The tile origins per axis are either
    given (`origins` = (z list, y list, x list), every tile inside the volume)
    or laid on a grid of `stride` (d, h, w) by `grid_axis`."""
    from . import pyramid_crop, pyramid_stitch_add, pyramid_stitch_clear, pyramid_stitch_finish
    N, D, H, W, C = x.shape
    K = head[0].shape[0]
    if origins is None:
        if stride is None:
            raise ValueError("give a stride or explicit tile origins")
        (zs, td), (ys, th), (xs, tw) = (grid_axis(e, t, s) for e, t, s in
                                        zip((D, H, W), tile, stride))
    else:
        td, th, tw = tile
        zs, ys, xs = (list(o) for o in origins)
        for ext, size, starts in ((D, td, zs), (H, th, ys), (W, tw, xs)):
            if not starts or min(starts) < 0 or max(starts) + size > ext:
                raise ValueError("tile origins must keep every tile inside the volume")
    out = torch.empty((N, D, H, W, K), dtype=torch.float32, device=x.device)
    acc = torch.empty((D, H, W, K), dtype=torch.float32, device=x.device)
    wsum = torch.empty((D, H, W), dtype=torch.float32, device=x.device)
    sub = torch.empty((1, td, th, tw, C), dtype=x.dtype, device=x.device)
    for n in range(N):
        pyramid_stitch_clear(acc, wsum, stream)
        for z0 in zs:
            for y0 in ys:
                for x0 in xs:
                    box = (z0, y0, x0, td, th, tw)
                    pyramid_crop(x, n, box, sub, stream)
                    p = network_forward(sub, layers, fcs, head, ws=ws, stream=stream,
                                        norms=norms)["p"]
                    pyramid_stitch_add(p.view(td, th, tw, K), box, acc, wsum, sigma_scale,
                                       stream)
        pyramid_stitch_finish(acc, wsum, out[n], stream)
    return out

