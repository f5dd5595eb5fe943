"""Timing cases of the sequence and checkpoint operators: layer norm over channels, the gated linear scan along an axis and
8-bit activation checkpoints.

A case is one call (or the forward and backward calls of one training step) on seeded inputs. `run` computes it in plain torch
operations or, with `own` set, through the package's entry points. `listed()` gives the fixed cases, `draw(rng)` further ones of
the same ranges.
"""
import math

import torch

own = False     # True: run() calls the package's operators

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-5
BLOCK = 64      # elements that share a scale (bf16) in an 8-bit checkpoint
SMALL = 2.0 ** -119     # a block whose largest magnitude is below this is held as zeros
RUN = 16        # steps between the states that a training scan keeps

# kind "norm": M rows of C channels; "train" adds the backward, "ckpt" keeps the forward's input in 8 bits for it.
# kind "scan": B sequences of T steps of I channels; "reverse" sweeps from the last step; "ragged" gives each sequence a length
#   of its own; "state" passes a state in and takes the last one out (and, in training, their gradients); "train" and "ckpt" as above.
# kind "ckpt": n values held in 8 bits and taken back.


def listed():
    return [
        # the rows of one decoding step of a batch of eight: launch latency
        {"name": "norm-token", "kind": "norm", "M": 8, "C": 1024, "dtype": "bf16", "train": False, "ckpt": False},
        # training over a whole MR volume behind the first layer (48 x 240 x 240 voxels of 16 units)
        {"name": "norm-mr", "kind": "norm", "M": 2764800, "C": 16, "dtype": "f32", "train": True, "ckpt": False},
        # the paper network's odd FC width over a sub-volume, its input held in 8 bits
        {"name": "norm-odd-ckpt", "kind": "norm", "M": 360000, "C": 45, "dtype": "f32", "train": True, "ckpt": True},
        # training over wide rows, as in a language model's block
        {"name": "norm-wide", "kind": "norm", "M": 8192, "C": 4096, "dtype": "bf16", "train": True, "ckpt": False},
        # one step of a batch of sixteen with the state carried: launch latency
        {"name": "scan-token", "kind": "scan", "B": 16, "T": 1, "I": 2048, "dtype": "bf16", "reverse": False, "ragged": False,
         "state": True, "train": False, "ckpt": False},
        # training along x of a whole MR volume, from the far side (x- sweep), 16 units
        {"name": "scan-mr-x", "kind": "scan", "B": 11520, "T": 240, "I": 16, "dtype": "f32", "reverse": True, "ragged": False,
         "state": False, "train": True, "ckpt": False},
        # one long sequence, inference
        {"name": "scan-long", "kind": "scan", "B": 1, "T": 65536, "I": 1024, "dtype": "bf16", "reverse": False, "ragged": False,
         "state": True, "train": False, "ckpt": False},
        # training on two long sequences
        {"name": "scan-step", "kind": "scan", "B": 2, "T": 8192, "I": 2048, "dtype": "f32", "reverse": False, "ragged": False,
         "state": False, "train": True, "ckpt": False},
        # training on a padded batch of odd sizes, the gates and inputs held in 8 bits
        {"name": "scan-ragged-ckpt", "kind": "scan", "B": 7, "T": 1531, "I": 333, "dtype": "bf16", "reverse": True, "ragged": True,
         "state": True, "train": True, "ckpt": True},
        # the activations of a smoke-size layer: launch latency, a last block cut short
        {"name": "ckpt-small", "kind": "ckpt", "n": 12345, "dtype": "f32"},
        # the gates that a layer of 16 units saves for two 8 x 64 x 64 training cubes
        {"name": "ckpt-gates", "kind": "ckpt", "n": 25165824, "dtype": "f32"},
        # the activations of a long bf16 batch
        {"name": "ckpt-bf16", "kind": "ckpt", "n": 134217728, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "scan", "scan", "ckpt"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "norm":
        C = rng.choice([_log_int(rng, 1, 8192), rng.choice([16, 32, 64, 256, 1024, 2048])])
        M = _log_int(rng, 1, max(1, 30000000 // C))
        train = rng.random() < 0.7
        return {"kind": "norm", "M": M, "C": C, "dtype": dtype, "train": train, "ckpt": train and rng.random() < 0.5}
    if kind == "scan":
        T = rng.choice([_log_int(rng, 1, 65536), _log_int(rng, 16, 2048)])
        I = rng.choice([_log_int(rng, 1, 4096), rng.choice([16, 32, 64, 512, 1024, 2048])])
        I = min(I, max(1, 30000000 // T))
        B = _log_int(rng, 1, max(1, 30000000 // (T * I)))
        B = min(B, 20000)
        train = rng.random() < 0.6
        return {"kind": "scan", "B": B, "T": T, "I": I, "dtype": dtype, "reverse": rng.random() < 0.5,
                "ragged": 1 < T <= 8192 and rng.random() < 0.4, "state": rng.random() < 0.5, "train": train,
                "ckpt": train and rng.random() < 0.4}
    return {"kind": "ckpt", "n": _log_int(rng, 1000, 100000000), "dtype": dtype}


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(gen, shape, dtype, scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale + shift).to(DT[dtype])


def prepare(case, seed):
    gen = _generator(seed)
    dt, s = case["dtype"], {"case": case}
    if case["kind"] == "norm":
        M, C = case["M"], case["C"]
        # activations: a common level, channels of their own level
        s["x"] = (torch.randn((M, C), generator=gen, device="cuda") * 0.8 +
                  torch.randn(C, generator=gen, device="cuda") * 0.5 + 0.2).to(DT[dt])
        s["gamma"] = _normal(gen, C, dt, 0.2, 1.0)
        s["beta"] = _normal(gen, C, dt, 0.1)
        if case["train"]:
            s["dy"] = _normal(gen, (M, C), dt, 0.1)
    elif case["kind"] == "scan":
        B, T, I = case["B"], case["T"], case["I"]
        # gates that keep about 0.5 to 0.99 of the state
        s["g"] = _normal(gen, (B, T, I), dt, 1.5, 2.0)
        s["u"] = _normal(gen, (B, T, I), dt)
        s["lengths"] = None
        if case["ragged"]:
            # lengths from nothing to all, the longest as long as the batch
            s["lengths"] = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
            s["lengths"][B // 2] = T
        s["h0"] = _normal(gen, (B, I), "f32") if case["state"] else None
        if case["train"]:
            s["dh"] = _normal(gen, (B, T, I), dt, 0.1)
            s["dhT"] = _normal(gen, (B, I), "f32", 0.1) if case["state"] else None
    else:
        # gate-like and input-like activations; runs of small values among them
        x = torch.tanh(torch.randn(case["n"], generator=gen, device="cuda"))
        x[: case["n"] // 3] *= 0.01
        s["x"] = x.to(DT[dt])
    return s


def work(case):
    e = SIZE[case["dtype"]]
    codes = 1 + 2 / BLOCK
    if case["kind"] == "norm":
        n, C = case["M"] * case["C"], case["C"]
        b, f = 2 * e * n + 2 * e * C, 8 * n
        if case["train"]:
            # the backward reads dy and the input (or its codes), writes dx and the weights' gradients
            b += 2 * e * n + (2 * codes if case["ckpt"] else e) * n + 16 * case["M"] + 8 * C
            f += 14 * n
        return {"bytes": b, "flops": f}
    if case["kind"] == "scan":
        n, cols = case["B"] * case["T"] * case["I"], case["B"] * case["I"]
        b, f = 3 * e * n, 8 * n
        if case["state"]:
            b += 8 * cols
        if case["train"]:
            states = 4 * cols * -(-case["T"] // RUN)
            b += 2 * states + 3 * e * n + (4 * codes if case["ckpt"] else 2 * e) * n + (8 * cols if case["state"] else 0)
            f += 20 * n
        return {"bytes": b, "flops": f}
    return {"bytes": 2 * (e + codes) * case["n"], "flops": 4 * case["n"]}


# ------------------------------------------------------------------ plain forms

def _through_8_bits(x):
    """fp32 values that the 8-bit checkpoint of x stands for (code * scale has 15 bits: exact)."""
    n = x.numel()
    v = torch.zeros(-(-n // BLOCK) * BLOCK, device=x.device)
    v[:n] = x.reshape(-1).float()
    v = v.view(-1, BLOCK)
    top = v.abs().amax(1, keepdim=True)
    # the smallest bf16 number that is at least top / 127: the one at or below, or the next (products of 8 and 7 bits are exact)
    low = ((top / 127).view(torch.int32) >> 16 << 16).view(torch.float32)
    scale = torch.where(low * 127 < top, ((low.view(torch.int32) >> 16) + 1 << 16).view(torch.float32), low)
    scale = torch.where(top < SMALL, torch.zeros_like(top), scale)
    # the quotient in 64 bits: in 32 it may fall on a tie that the true one misses
    code = torch.where(scale > 0, torch.round(v.double() / scale.double()).float(), torch.zeros_like(v))
    return (code * scale).reshape(-1)[:n].view(x.shape)


def _plain_norm(s):
    case, x = s["case"], s["x"]
    C, gamma = case["C"], s["gamma"].float()

    def parts(v):
        return (v - mean) * rstd

    xf = x.float()
    mean = xf.sum(1, keepdim=True) / C
    d = xf - mean
    rstd = 1 / torch.sqrt((d * d).sum(1, keepdim=True) / C + EPS)
    y = (parts(xf) * gamma + s["beta"].float()).to(x.dtype)
    if not case["train"]:
        return [y]
    xhat = parts(_through_8_bits(x)) if case["ckpt"] else parts(xf)
    dy = s["dy"].float()
    a = dy * gamma
    dx = rstd * (a - a.sum(1, keepdim=True) / C - xhat * ((a * xhat).sum(1, keepdim=True) / C))
    return [y, dx.to(x.dtype), (dy * xhat).sum(0), dy.sum(0)]


def _prefix(a, b):
    """The recurrence v_s = a_s v_{s-1} + b_s along axis 1 from v = 0, and the products of a, by doubling: after the pass
    with distance d a position holds the composition of its 2 d last steps."""
    d = 1
    while d < a.shape[1]:
        b = torch.cat([b[:, :d], b[:, d:] + a[:, d:] * b[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return a, b


def _order(case, lengths, device):
    """Index [B][T] of the step at each sweep position (and of the position of each step: it is its own inverse), and which
    positions a sequence has."""
    pos = torch.arange(case["T"], device=device)[None, :]
    n = torch.full((case["B"], 1), case["T"], device=device) if lengths is None else lengths.long()[:, None]
    live = pos < n
    return torch.where(live, n - 1 - pos, pos) if case["reverse"] else pos.expand(case["B"], -1), live[:, :, None]


def _along(v, order):
    return torch.gather(v, 1, order[:, :, None].expand(-1, -1, v.shape[2]))


def _plain_scan(s):
    case, dtype = s["case"], s["g"].dtype
    B, T, I = case["B"], case["T"], case["I"]
    order, live = _order(case, s["lengths"], s["g"].device)
    zero, one = torch.zeros((), device=s["g"].device), torch.ones((), device=s["g"].device)
    h0 = s["h0"] if case["state"] else torch.zeros((B, I), device=s["g"].device)

    def gates(g, u):
        g, u = _along(g.float(), order), _along(u.float(), order)
        keep, take = torch.sigmoid(g), torch.sigmoid(-g)
        return torch.where(live, keep, one), torch.where(live, take, zero), torch.where(live, u, zero)

    keep, take, u = gates(s["g"], s["u"])
    prod, part = _prefix(keep, take * u)
    h = part + prod * h0[:, None]
    out = [_along(torch.where(live, h, zero), order).to(dtype)]
    if case["state"]:
        out.append(h[:, -1].contiguous())
    if not case["train"]:
        return out
    before = torch.cat([h0[:, None], h[:, :-1]], 1)
    if case["ckpt"]:
        # the backward has the values of the 8-bit checkpoints and the true states before every RUN-th step
        keep, take, u = gates(_through_8_bits(s["g"]), _through_8_bits(s["u"]))
        runs = -(-T // RUN)
        fill = runs * RUN - T

        def cut(v, value):
            return torch.cat([v, torch.full((B, fill, I), value, device=v.device)], 1).view(B * runs, RUN, I)

        p, q = _prefix(cut(keep, 1.0), cut(take * u, 0.0))
        at = before[:, ::RUN].reshape(B * runs, 1, I)
        before = torch.cat([at, q[:, :-1] + p[:, :-1] * at], 1).view(B, runs * RUN, I)[:, :T]
    dh = torch.where(live, _along(s["dh"].float(), order), zero)
    dhT = s["dhT"] if case["state"] else torch.zeros((B, I), device=dh.device)
    # G_s = dh_s + keep_{s+1} G_{s+1}: the same recurrence from the other end
    later = torch.cat([keep[:, 1:], torch.ones((B, 1, I), device=keep.device)], 1)
    prod, part = _prefix(later.flip(1), dh.flip(1))
    G = (part + prod * dhT[:, None]).flip(1)
    dg = torch.where(live, G * (before - u) * keep * take, zero)
    du = torch.where(live, G * take, zero)
    out += [_along(dg, order).to(dtype), _along(du, order).to(dtype)]
    if case["state"]:
        out.append(keep[:, 0] * G[:, 0])
    return out


# --------------------------------------------------------- the package's entry points

def _own_norm(s):
    import paper_1506_07452_amd as P
    case, x = s["case"], s["x"]
    y = torch.empty_like(x)
    if not case["train"]:
        P.pyramid_layer_norm_forward(x, s["gamma"], s["beta"], y, eps=EPS)
        return [y]
    stats = torch.empty((case["M"], 2), dtype=torch.float32, device=x.device)
    kept, scale = x, None
    if case["ckpt"]:
        kept, scale = P.checkpoint8_empty(x)
    P.pyramid_layer_norm_forward(x, s["gamma"], s["beta"], y, stats, kept if case["ckpt"] else None, scale, eps=EPS)
    dx = torch.empty_like(x)
    dgamma, dbeta = (torch.empty(case["C"], dtype=torch.float32, device=x.device) for _ in range(2))
    P.pyramid_layer_norm_backward(kept, s["gamma"], stats, s["dy"], dx, dgamma, dbeta, xscale=scale)
    return [y, dx, dgamma, dbeta]


def _own_scan(s):
    import paper_1506_07452_amd as P
    case, g, u = s["case"], s["g"], s["u"]
    B, T, I = case["B"], case["T"], case["I"]
    h = torch.empty_like(g)
    hT = torch.empty((B, I), dtype=torch.float32, device=g.device) if case["state"] else None
    saved = None
    if case["train"]:
        saved = torch.empty(P.pyramid_scan_saved_size(B, T, I), dtype=torch.uint8, device=g.device)
    P.pyramid_scan_forward(g, u, h, reverse=case["reverse"], lengths=s["lengths"], h0=s["h0"], hT=hT, saved=saved)
    out = [h] + ([hT] if case["state"] else [])
    if not case["train"]:
        return out
    gscale = uscale = None
    if case["ckpt"]:
        g, gscale = P.checkpoint8_empty(s["g"])
        P.pyramid_checkpoint8_pack(s["g"], g, gscale)
        u, uscale = P.checkpoint8_empty(s["u"])
        P.pyramid_checkpoint8_pack(s["u"], u, uscale)
    dg, du = torch.empty_like(h), torch.empty_like(h)
    dh0 = torch.empty((B, I), dtype=torch.float32, device=h.device) if case["state"] else None
    P.pyramid_scan_backward(g, u, saved, s["dh"], dg, du, reverse=case["reverse"], lengths=s["lengths"], dhT=s["dhT"], dh0=dh0,
                            gscale=gscale, uscale=uscale)
    return out + [dg, du] + ([dh0] if case["state"] else [])


def _own_ckpt(s):
    import paper_1506_07452_amd as P
    q, scale = P.checkpoint8_empty(s["x"])
    P.pyramid_checkpoint8_pack(s["x"], q, scale)
    back = torch.empty_like(s["x"])
    P.pyramid_checkpoint8_unpack(q, scale, back)
    return [back]


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"norm": _own_norm, "scan": _own_scan, "ckpt": _own_ckpt}[kind](state)
    if kind == "ckpt":
        return [_through_8_bits(state["x"]).to(state["x"].dtype)]
    return _plain_norm(state) if kind == "norm" else _plain_scan(state)


# ------------------------------------------------------------- the definition, in 64 bits

def _codes64(x):
    """Values of the 8-bit checkpoint of a tensor: blocks of BLOCK elements in order, the scale the smallest number of 8 significant
    bits that is at least a 127th of the largest magnitude, codes to the nearest, ties to the even one."""
    n = x.numel()
    flat = torch.nn.functional.pad(x.reshape(-1).double(), (0, -n % BLOCK)).reshape(-1, BLOCK)
    top = flat.abs().max(dim=1, keepdim=True).values
    # by a tensor: a division by a number is a product with its rounded inverse, which misses quotients that are exact
    scale = top / torch.full_like(top, 127.0)
    scale = ((scale.view(torch.int64) + (1 << 45) - 1) >> 45 << 45).view(torch.float64)     # up to 8 significant bits
    scale[top < SMALL] = 1.0
    value = (flat / scale).round() * scale
    value[(top < SMALL).expand_as(value)] = 0.0
    return value.reshape(-1)[:n].reshape(x.shape)


def _exact_norm(s):
    case, x = s["case"], s["x"].double()
    var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
    std = (var + EPS).sqrt()
    gamma = s["gamma"].double()
    y = (x - mean) / std * gamma + s["beta"].double()
    if not case["train"]:
        return [y]
    z = ((_codes64(s["x"]) if case["ckpt"] else x) - mean) / std
    dy = s["dy"].double()
    w = dy * gamma
    dx = (w - w.mean(1, keepdim=True) - z * (w * z).mean(1, keepdim=True)) / std
    return [y, dx, (dy * z).sum(0), dy.sum(0)]


def _exact_scan(s):
    case = s["case"]
    B, T, I = case["B"], case["T"], case["I"]
    dev = s["g"].device
    rows = torch.arange(B, device=dev)

    def step_of(p):
        # the step at sweep position p (of each sequence, where they differ in length) and where there is one
        if s["lengths"] is None:
            return (T - 1 - p if case["reverse"] else p), None
        n = s["lengths"].long()
        has = p < n
        return torch.where(has, (n - 1 - p) if case["reverse"] else torch.full_like(n, p), torch.full_like(n, p)), has[:, None]

    def take(v, at):
        return v[:, at].double() if s["lengths"] is None else v[rows, at].double()

    def put(v, at, value):
        v[(slice(None) if s["lengths"] is None else rows), at] = value

    def where(has, value, other):
        return value if has is None else torch.where(has, value, other)

    state = s["h0"].double() if case["state"] else torch.zeros((B, I), dtype=torch.float64, device=dev)
    h = torch.zeros((B, T, I), dtype=torch.float64, device=dev)
    g, u = s["g"], s["u"]
    gq, uq = (_codes64(g), _codes64(u)) if case["train"] and case["ckpt"] else (g, u)
    before = torch.zeros_like(h) if case["train"] else None     # the state that the backward has, by sweep position
    held = state
    for p in range(T):
        at, has = step_of(p)
        f = 1 / (1 + torch.exp(-take(g, at)))
        if case["train"]:
            if p % RUN == 0 or not case["ckpt"]:
                held = state
            before[:, p] = held
            if case["ckpt"]:
                fq = 1 / (1 + torch.exp(-take(gq, at)))
                held = where(has, fq * held + (1 - fq) * take(uq, at), held)
        state = where(has, f * state + (1 - f) * take(u, at), state)
        put(h, at, where(has, state, torch.zeros_like(state)))
    out = [h] + ([state] if case["state"] else [])
    if not case["train"]:
        return out
    G = s["dhT"].double() if case["state"] else torch.zeros((B, I), dtype=torch.float64, device=dev)
    dg, du = torch.zeros_like(h), torch.zeros_like(h)
    for p in range(T - 1, -1, -1):
        at, has = step_of(p)
        f = 1 / (1 + torch.exp(-take(gq, at)))
        G = where(has, G + take(s["dh"], at), G)
        put(dg, at, where(has, G * (before[:, p] - take(uq, at)) * f * (1 - f), torch.zeros_like(G)))
        put(du, at, where(has, G * (1 - f), torch.zeros_like(G)))
        G = where(has, G * f, G)
    return out + [dg, du] + ([G] if case["state"] else [])


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "ckpt":
        return [_codes64(s["x"])]
    return _exact_norm(s) if case["kind"] == "norm" else _exact_scan(s)
