"""Timing cases of a selective-scan block and its update: the causal convolution, the selective state space scan, group norm
with an activation over channels-last volumes, and AdamW over many tensors with moments in 32 or 8 bits.

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
KEEP = 64       # steps between the states that a training scan keeps
BLOCK = 256     # elements that share the scales of 8-bit moments
LR, BETAS, ADAM_EPS, DECAY = 1e-3, (0.9, 0.999), 1e-8, 0.01

# kind "conv": B sequences of T steps of I channels, K taps, SiLU; the input is half of a row of 2 I channels. "state" passes the
#   last inputs in and out; "reverse" sweeps from the last step; "ragged" gives each sequence a length; "train" adds the backward.
# kind "scan": the same with S states a channel; B and C are slices of one projection's rows, "gate" multiplies by SiLU(z), z the
#   second half of the convolution's row of 2 I channels.
# kind "norm": N volumes of V voxels of C channels in G groups, "act" none or silu.
# kind "adamw": tensors of the `sizes`, gradients in "dtype" (with bf16, a bf16 copy of the parameters is written too), moments in
#   "bits"; "clip" scales the gradients by a number on the device.


def listed():
    return [
        # one step of a batch of sixteen: launch latency
        {"name": "conv-token", "kind": "conv", "B": 16, "T": 1, "I": 2048, "K": 4, "dtype": "bf16", "reverse": False,
         "ragged": False, "state": True, "train": False},
        # training on two sequences
        {"name": "conv-step", "kind": "conv", "B": 2, "T": 8192, "I": 2048, "K": 4, "dtype": "bf16", "reverse": False,
         "ragged": False, "state": False, "train": True},
        # one step of a batch of sixteen with the state carried in place
        {"name": "scan-token", "kind": "scan", "B": 16, "T": 1, "I": 2048, "S": 16, "dtype": "bf16", "reverse": False,
         "ragged": False, "state": True, "gate": True, "train": False},
        # one long prompt, its state kept for the steps that follow
        {"name": "scan-prompt", "kind": "scan", "B": 1, "T": 16384, "I": 1024, "S": 16, "dtype": "bf16", "reverse": False,
         "ragged": False, "state": True, "gate": True, "train": False},
        # training on two sequences
        {"name": "scan-step", "kind": "scan", "B": 2, "T": 4096, "I": 2048, "S": 16, "dtype": "bf16", "reverse": False,
         "ragged": False, "state": False, "gate": True, "train": True},
        # training along x of a whole MR volume (48 x 240 x 240 voxels of 16 units), from the far side
        {"name": "scan-mr-x", "kind": "scan", "B": 11520, "T": 240, "I": 16, "S": 16, "dtype": "f32", "reverse": True,
         "ragged": False, "state": False, "gate": False, "train": True},
        # training on a padded batch of odd sizes
        {"name": "scan-ragged", "kind": "scan", "B": 5, "T": 1531, "I": 333, "S": 5, "dtype": "bf16", "reverse": True,
         "ragged": True, "state": True, "gate": True, "train": True},
        # a small 2D patch, inference: launch latency
        {"name": "norm-patch", "kind": "norm", "N": 1, "V": 4096, "C": 32, "G": 8, "dtype": "bf16", "act": "silu", "train": False},
        # training over a whole MR volume behind the first layer
        {"name": "norm-mr", "kind": "norm", "N": 1, "V": 2764800, "C": 16, "G": 4, "dtype": "f32", "act": "silu", "train": True},
        # training over a batch of eight 64 x 64 x 64 cubes of 64 units
        {"name": "norm-cubes", "kind": "norm", "N": 8, "V": 262144, "C": 64, "G": 8, "dtype": "bf16", "act": "silu", "train": True},
        # the two-layer network's parameters (16 and 32 units, 3 input channels)
        {"name": "adamw-net", "kind": "adamw", "sizes": "10368,55296,384,512,32,221184,221184,768,2048,64,256,4", "dtype": "f32",
         "bits": 32, "clip": True},
        # the parameters of a large network, bf16 gradients and weights, moments in 8 bits
        {"name": "adamw-large-8", "kind": "adamw",
         "sizes": "33554432,16777216,8388608,4194304,2097152,1048576,65536,2048,2048,45,333,7", "dtype": "bf16", "bits": 8,
         "clip": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["conv", "scan", "scan", "scan", "norm", "norm", "adamw"])
    dtype = rng.choice(["f32", "bf16"])
    if kind in ("conv", "scan"):
        S = rng.choice([16, 16, 8, _log_int(rng, 1, 64)])
        most = 25000000 if kind == "conv" else 250000000 // (S + 4)
        T = rng.choice([1, _log_int(rng, 2, 8192), _log_int(rng, 16, 2048)])
        I = min(rng.choice([_log_int(rng, 1, 4096), rng.choice([16, 32, 64, 512, 1024, 2048])]), max(1, most // T))
        B = min(_log_int(rng, 1, max(1, most // (T * I))), 12000)
        case = {"kind": kind, "B": B, "T": T, "I": I, "dtype": dtype, "reverse": rng.random() < 0.4,
                "ragged": T > 1 and rng.random() < 0.4, "state": T == 1 or rng.random() < 0.5,
                "train": T > 1 and rng.random() < 0.6}
        return dict(case, K=rng.choice([4, 4, 2, 3, 8])) if kind == "conv" else dict(case, S=S, gate=rng.random() < 0.7)
    if kind == "norm":
        G = _log_int(rng, 1, 32)
        C = G * _log_int(rng, 1, 64)
        N = _log_int(rng, 1, 64)
        return {"kind": "norm", "N": N, "V": _log_int(rng, 1, max(1, 40000000 // (N * C))), "C": C, "G": G, "dtype": dtype,
                "act": rng.choice(["none", "silu"]), "train": rng.random() < 0.7}
    sizes = [_log_int(rng, 1, 4000000) for _ in range(_log_int(rng, 1, 12))]
    return {"kind": "adamw", "sizes": ",".join(str(n) for n in sizes), "dtype": dtype, "bits": rng.choice([8, 32]),
            "clip": rng.random() < 0.5}


def _normal(gen, shape, dtype="f32", scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale + shift).to(DT[dtype])


def _lengths(gen, B, T):
    # from nothing to all, the longest as long as the batch
    n = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    n[B // 2] = T
    return n


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, s = case["dtype"], {"case": case}
    if case["kind"] == "conv":
        B, T, I, K = case["B"], case["T"], case["I"], case["K"]
        s["x"] = _normal(gen, (B, T, 2 * I), dt)[:, :, :I]
        s["w"] = _normal(gen, (I, K), dt, K ** -0.5)
        s["bias"] = _normal(gen, I, dt, 0.1)
        s["lengths"] = _lengths(gen, B, T) if case["ragged"] else None
        s["state"] = _normal(gen, (B, K - 1, I), dt) if case["state"] else None
        if case["train"]:
            s["dy"] = _normal(gen, (B, T, I), dt, 0.1)
            s["dstate"] = _normal(gen, (B, K - 1, I), "f32", 0.1) if case["state"] else None
    elif case["kind"] == "scan":
        B, T, I, S = case["B"], case["T"], case["I"], case["S"]
        s["u"] = _normal(gen, (B, T, I), dt)
        s["delta"] = _normal(gen, (B, T, I), dt, 0.5)
        # steps of 0.001 to 0.1 behind the softplus, decays of 1 to S
        step = torch.exp(torch.rand(I, generator=gen, device="cuda") * math.log(100.0) + math.log(0.001))
        s["dbias"] = torch.log(torch.expm1(step))
        s["A"] = -torch.exp(torch.randn((I, S), generator=gen, device="cuda") * 0.2 +
                            torch.log(torch.arange(1, S + 1, device="cuda", dtype=torch.float32)))
        s["D"] = _normal(gen, I, "f32", 0.2, 1.0)
        rows = _normal(gen, (B, T, 2 * S), dt)
        s["B"], s["C"] = rows[:, :, :S], rows[:, :, S:]
        s["z"] = _normal(gen, (B, T, 2 * I), dt)[:, :, I:] if case["gate"] else None
        s["lengths"] = _lengths(gen, B, T) if case["ragged"] else None
        s["h0"] = _normal(gen, (B, I, S)) if case["state"] else None
        if case["train"]:
            s["dy"] = _normal(gen, (B, T, I), dt, 0.1)
            s["dhT"] = _normal(gen, (B, I, S), "f32", 0.1) if case["state"] else None
    elif case["kind"] == "norm":
        N, V, C = case["N"], case["V"], case["C"]
        # activations: a common level, channels and volumes of their own level
        s["x"] = (torch.randn((N, V, C), generator=gen, device="cuda") * 0.8 +
                  torch.randn((N, 1, C), generator=gen, device="cuda") * 0.5 + 0.2).to(DT[dt])
        s["gamma"] = _normal(gen, C, dt, 0.2, 1.0)
        s["beta"] = _normal(gen, C, dt, 0.1)
        if case["train"]:
            s["dy"] = _normal(gen, (N, V, C), dt, 0.1)
    else:
        sizes = [int(n) for n in case["sizes"].split(",")]
        s["p"] = [_normal(gen, n, "f32", 0.05) for n in sizes]
        s["g"] = [_normal(gen, n, dt, 0.01) for n in sizes]
        s["copies"] = [p.to(torch.bfloat16) for p in s["p"]] if dt == "bf16" else None
        s["t"] = 100 + seed % 1000
        s["scale"] = torch.rand(1, generator=gen, device="cuda") * 0.5 + 0.5 if case["clip"] else None
        if case["bits"] == 32:
            s["m"] = [_normal(gen, n, "f32", 0.003) for n in sizes]
            s["v"] = [_normal(gen, n, "f32", 0.01).square() for n in sizes]
        else:
            s["m"], s["v"], s["ms"], s["vs"] = [], [], [], []
            for n in sizes:
                m = torch.randint(60, 121, (n,), generator=gen, device="cuda", dtype=torch.uint8)
                s["m"].append(m | torch.randint(0, 2, (n,), generator=gen, device="cuda", dtype=torch.uint8) << 7)
                s["v"].append(torch.randint(190, 249, (n,), generator=gen, device="cuda", dtype=torch.uint8))
                blocks = -(-n // BLOCK)
                s["ms"].append(torch.exp(_normal(gen, blocks, "f32", 0.3, math.log(0.01))))
                s["vs"].append(torch.exp(_normal(gen, blocks, "f32", 0.3, math.log(0.0003))))
    return s


def work(case):
    e = SIZE[case["dtype"]]
    if case["kind"] == "conv":
        n, I, K = case["B"] * case["T"] * case["I"], case["I"], case["K"]
        state = case["B"] * (K - 1) * I
        b, f = 2 * e * n + e * I * (K + 1) + (2 * e * state if case["state"] else 0), n * (2 * K + 6)
        if case["train"]:
            b += 3 * e * n + 4 * I * (K + 1) + (8 * state if case["state"] else 0)
            f += n * (6 * K + 12)
        return {"bytes": b, "flops": f}
    if case["kind"] == "scan":
        B, T, I, S = case["B"], case["T"], case["I"], case["S"]
        n, rows, cols = B * T * I, B * T * S, B * I * S
        ins = 3 if case["gate"] else 2
        b, f = (ins + 1) * e * n + 2 * e * rows + 4 * I * (S + 2), n * (7 * S + 15)
        if case["state"]:
            b += 8 * cols
        if case["train"]:
            b += 2 * 4 * cols * -(-T // KEEP) + (ins + 1 + ins) * e * n + 4 * e * rows + 4 * I * (S + 2) * 2
            b += 8 * cols if case["state"] else 0
            f += n * (22 * S + 30)
        return {"bytes": b, "flops": f}
    if case["kind"] == "norm":
        n = case["N"] * case["V"] * case["C"]
        return {"bytes": (5 if case["train"] else 2) * e * n, "flops": (30 if case["train"] else 10) * n}
    n = sum(int(k) for k in case["sizes"].split(","))
    b = e + 8 + (2 if case["dtype"] == "bf16" else 0)
    # 8-bit moments: codes read and written, and the values that they stand for given back
    b += 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 8
    return {"bytes": b * n, "flops": 20 * n}


# ------------------------------------------------------------------ plain forms

def _prefix(a, b):
    """The recurrence v_s = a_s v_{s-1} + b_s along axis 1 from v = 0, and the products of a, by doubling: after the pass
    with distance d a position holds the composition of its 2 d last steps."""
    d = 1
    while d < a.shape[1]:
        b = torch.cat([b[:, :d], b[:, d:] + a[:, d:] * b[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return a, b


class _Order:
    """Between steps and sweep positions (the map is its own inverse), and which positions a sequence has."""

    def __init__(self, case, lengths, device):
        self.flip = case["reverse"] and lengths is None
        self.index = self.live = None
        if lengths is not None:
            pos = torch.arange(case["T"], device=device)[None, :]
            n = lengths.long()[:, None]
            self.live = (pos < n)[:, :, None]
            self.index = torch.where(pos < n, n - 1 - pos, pos)[:, :, None] if case["reverse"] else None

    def along(self, v):
        if self.index is not None:
            return torch.gather(v, 1, self.index.expand(-1, -1, v.shape[2]))
        return v.flip(1) if self.flip else v

    def have(self, v):
        return v if self.live is None else torch.where(self.live, v, torch.zeros((), dtype=v.dtype, device=v.device))


def _plain_conv(s):
    case, dtype = s["case"], s["x"].dtype
    B, T, I, K = case["B"], case["T"], case["I"], case["K"]
    order = _Order(case, s["lengths"], s["x"].device)
    before = s["state"] if case["state"] else torch.zeros((B, K - 1, I), dtype=dtype, device=s["x"].device)
    xs = torch.cat([before.float(), order.have(order.along(s["x"].float()))], 1)
    taps = xs.unfold(1, K, 1)
    w = s["w"].float()
    a = (taps * w).sum(-1) + s["bias"].float()
    sg = torch.sigmoid(a)
    out = [order.along(order.have(a * sg)).to(dtype)]
    n = s["lengths"].long() if case["ragged"] else torch.full((B,), T, device=xs.device)
    last = (n[:, None] + torch.arange(K - 1, device=xs.device))[:, :, None].expand(-1, -1, I)
    if case["state"]:
        out.append(torch.gather(xs, 1, last).to(dtype))
    if not case["train"]:
        return out
    da = order.have(order.along(s["dy"].float())) * sg * (1 + a * (1 - sg))
    dxs = (torch.nn.functional.pad(da, (0, 0, K - 1, K - 1)).unfold(1, K, 1) * w.flip(1)).sum(-1)
    if case["state"]:
        dxs = dxs.scatter_add(1, last, s["dstate"])
    out += [order.along(order.have(dxs[:, K - 1:])).to(dtype),
            (da[..., None] * taps).double().sum((0, 1)).float(), da.double().sum((0, 1)).float()]
    return out + ([dxs[:, :K - 1].contiguous()] if case["state"] else [])


def _plain_scan(s):
    case, dtype, dev = s["case"], s["u"].dtype, s["u"].device
    B, I, S = case["B"], case["I"], case["S"]
    order = _Order(case, s["lengths"], dev)

    def get(v):
        return order.have(order.along(v.float()))

    u, raw = get(s["u"]), order.along(s["delta"].float()) + s["dbias"]
    dt = order.have(raw.clamp(min=0) + torch.log1p(torch.exp(-raw.abs())))
    Bm, Cm = get(s["B"])[:, :, None], get(s["C"])[:, :, None]
    A, D = s["A"], s["D"]
    h0 = s["h0"] if case["state"] else torch.zeros((B, I, S), device=dev)
    a = torch.exp(dt[..., None] * A)
    prod, h = _prefix(a, (dt * u)[..., None] * Bm)
    h = h + prod * h0[:, None]
    del prod
    p = (h * Cm).sum(-1) + D * u
    if case["gate"]:
        z = get(s["z"])
        sg = torch.sigmoid(z)
    y = p * z * sg if case["gate"] else p
    out = [order.along(order.have(y)).to(dtype)] + ([h[:, -1].contiguous()] if case["state"] else [])
    if not case["train"]:
        return out
    dy = get(s["dy"])
    dp = dy * z * sg if case["gate"] else dy
    dhT = s["dhT"] if case["state"] else torch.zeros((B, I, S), device=dev)
    # G_s = C dp_s + a_{s+1} G_{s+1}: the same recurrence from the other end
    later = torch.cat([a[:, 1:], torch.ones((B, 1, I, S), device=dev)], 1)
    prod, G = _prefix(later.flip(1), (Cm * dp[..., None]).flip(1))
    G = (G + prod * dhT[:, None]).flip(1)
    del prod, later
    dC = (h * dp[..., None]).sum(2)
    h = torch.cat([h0[:, None], h[:, :-1]], 1)      # the states before
    dB = (G * (dt * u)[..., None]).sum(2)
    q = (G * Bm).sum(-1)
    dh0 = a[:, 0] * G[:, 0]
    h = G * a * h
    del G, a
    dA = (h * dt[..., None]).double().sum((0, 1)).float()
    draw_ = (u * q + (h * A).sum(-1)) * order.have(torch.sigmoid(raw))
    out += [order.along(order.have(dt * q + D * dp)).to(dtype), order.along(draw_).to(dtype), dA, order.along(dB).to(dtype),
            order.along(dC).to(dtype), (dp * u).double().sum((0, 1)).float(), draw_.double().sum((0, 1)).float()]
    if case["gate"]:
        out.append(order.along(order.have(dy * p * sg * (1 + z * (1 - sg)))).to(dtype))
    return out + ([dh0] if case["state"] else [])


def _plain_norm(s):
    case, x = s["case"], s["x"].float()
    N, V, C, G = case["N"], case["V"], case["C"], case["G"]
    gamma, beta = s["gamma"].float(), s["beta"].float()
    x = x.view(N, V, G, C // G)
    mean = x.double().mean((1, 3), keepdim=True)
    d = (x - mean.float()) - (mean - mean.float().double()).float()
    rstd = (1 / torch.sqrt((d * d).double().mean((1, 3), keepdim=True) + EPS)).float()
    xh = (d * rstd).view(N, V, C)
    v = xh * gamma + beta
    if case["act"] == "silu":
        sg = torch.sigmoid(v)
        y = v * sg
    else:
        y = v
    if not case["train"]:
        return [y.to(s["x"].dtype)]
    dv = s["dy"].float()
    if case["act"] == "silu":
        dv = dv * sg * (1 + v * (1 - sg))
    a = (dv * gamma).view(N, V, G, C // G)
    xg = xh.view(N, V, G, C // G)
    m1 = a.double().mean((1, 3), keepdim=True).float()
    m2 = (a * xg).double().mean((1, 3), keepdim=True).float()
    dx = (a - m1 - xg * m2) * rstd
    return [y.to(s["x"].dtype), dx.view(N, V, C).to(s["x"].dtype), (dv * xh).double().sum((0, 1)).float(),
            dv.double().sum((0, 1)).float()]


WORD = 0xffffffff


def _mix(x):
    """A 32-bit integer hash (xorshift-multiply: 16, 7feb352d, 15, 846ca68b, 16) of values below 2^32 held in int64."""
    x = ((x ^ (x >> 16)) * 0x7feb352d) & WORD
    x = ((x ^ (x >> 15)) * 0x846ca68b) & WORD
    return x ^ (x >> 16)


def _mix_number(x):
    return int(_mix(torch.tensor(x & WORD, dtype=torch.int64)))


def _table(bits, low, device):
    """Values of the codes 0 .. 127 or 255: `bits` bits of exponent that end at 2^0, three of mantissa, the lowest exponent's
    codes linear down to 0 (`low`: the exponent of codes 0 .. 15)."""
    k = torch.arange(8 << bits, device=device)
    return torch.where(k < 8, k.double() / 8, 1 + (k & 7).double() / 8) * torch.exp2((torch.clamp(k >> 3, min=1) - 1 + low).double())


def _wide(codes, scale, low):
    """The fp32 values of codes (signed where low is -14) of blocks with their scales."""
    k = codes.long()
    table = _table(4, -14, codes.device) if low == -14 else _table(5, -30, codes.device)
    value = table[k & 127] * torch.where(k > 127, -1.0, 1.0).double() if low == -14 else table[k]
    return (value * scale.double().repeat_interleave(BLOCK)[:codes.numel()]).float()


def _narrow(x, low, random):
    """Codes and scales of fp32 values; random: 16 random bits an element, as integers."""
    n = x.numel()
    bits = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    scale = bits.abs().amax(1)
    r = (bits.abs().double() / torch.where(scale > 0, scale, torch.ones_like(scale)).double()[:, None]).reshape(-1)[:n]
    # three bits of mantissa and 16 behind them of the ratio's, in 64 bits, with its exponent above them
    fine = (r.view(torch.int64) >> 33) - ((1023 + low - 1) << 19)
    linear = (r * 2.0 ** (19 - low)).long()
    code = (torch.where(r < 2.0 ** low, linear, fine) + random) >> 16
    if low == -14:
        code = code + torch.where((x < 0) & (code > 0), 128, 0)
    else:
        code = torch.where((r > 0) & (code == 0), torch.ones_like(code), code)
    return code.to(torch.uint8), scale


def _plain_adamw(s):
    case, eight = s["case"], s["case"]["bits"] == 8
    s["t"] += 1
    t, (b1, b2) = s["t"], BETAS
    c1, c2 = 1 / (1 - b1 ** t), 1 / (1 - b2 ** t)
    values = []
    for k, p in enumerate(s["p"]):
        g = s["g"][k].double()
        if s["scale"] is not None:
            g = g * s["scale"].double()
        m = _wide(s["m"][k], s["ms"][k], -14) if eight else s["m"][k]
        v = _wide(s["v"][k], s["vs"][k], -30) if eight else s["v"][k]
        m, v = (m.double() * b1 + g * (1 - b1)).float(), (v.double() * b2 + g * g * (1 - b2)).float()
        p -= LR * (m * c1 / (torch.sqrt(v * c2) + ADAM_EPS) + DECAY * p)
        if s["copies"] is not None:
            s["copies"][k].copy_(p)
        if eight:
            key = _mix_number(_mix_number(t) + k)
            random = _mix(torch.arange(p.numel(), device=p.device) ^ key)
            s["m"][k], s["ms"][k] = _narrow(m, -14, random & 0xffff)
            s["v"][k], s["vs"][k] = _narrow(v, -30, random >> 16)
            m, v = _wide(s["m"][k], s["ms"][k], -14), _wide(s["v"][k], s["vs"][k], -30)
        else:
            s["m"][k].copy_(m)
            s["v"][k].copy_(v)
        values.append((m, v))
    return [s["p"], values, s["copies"]]


# --------------------------------------------------------- the package's entry points

def _own_conv(s):
    import paper_1506_07452_amd as P
    case, x = s["case"], s["x"]
    B, T, I, K = case["B"], case["T"], case["I"], case["K"]
    y = torch.empty((B, T, I), dtype=x.dtype, device=x.device)
    after = torch.empty_like(s["state"]) if case["state"] else None
    P.pyramid_causal_conv_forward(x, s["w"], s["bias"], y, act="silu", reverse=case["reverse"], lengths=s["lengths"],
                                  state=s["state"], state_out=after)
    out = [y] + ([after] if case["state"] else [])
    if not case["train"]:
        return out
    dx = torch.empty_like(y)
    dw = torch.empty((I, K), dtype=torch.float32, device=x.device)
    db = torch.empty(I, dtype=torch.float32, device=x.device)
    before = torch.empty((B, K - 1, I), dtype=torch.float32, device=x.device) if case["state"] else None
    P.pyramid_causal_conv_backward(x, s["w"], s["bias"], s["dy"], dx, dw, db, act="silu", reverse=case["reverse"],
                                   lengths=s["lengths"], state=s["state"], dstate_out=s["dstate"], dstate=before)
    return out + [dx, dw, db] + ([before] if case["state"] else [])


def _own_scan(s):
    import paper_1506_07452_amd as P
    case, u = s["case"], s["u"]
    B, T, I, S = case["B"], case["T"], case["I"], case["S"]
    how = dict(D=s["D"], z=s["z"], delta_bias=s["dbias"], softplus=True, reverse=case["reverse"], lengths=s["lengths"])
    y = torch.empty_like(u)
    hT = torch.empty((B, I, S), dtype=torch.float32, device=u.device) if case["state"] else None
    saved = None
    if case["train"]:
        saved = torch.empty(P.pyramid_selective_scan_saved_size(B, T, I, S), dtype=torch.uint8, device=u.device)
    P.pyramid_selective_scan_forward(u, s["delta"], s["A"], s["B"], s["C"], y, h0=s["h0"], hT=hT, saved=saved, **how)
    out = [y] + ([hT] if case["state"] else [])
    if not case["train"]:
        return out
    du, ddelta = torch.empty_like(u), torch.empty_like(u)
    dB, dC = (torch.empty((B, T, S), dtype=u.dtype, device=u.device) for _ in range(2))
    dA = torch.empty_like(s["A"])
    dD, dbias = torch.empty_like(s["D"]), torch.empty_like(s["D"])
    dz = torch.empty_like(u) if case["gate"] else None
    dh0 = torch.empty_like(s["h0"]) if case["state"] else None
    P.pyramid_selective_scan_backward(u, s["delta"], s["A"], s["B"], s["C"], saved, s["dy"], du, ddelta, dA, dB, dC, dD=dD,
                                      dz=dz, ddelta_bias=dbias, dhT=s["dhT"], dh0=dh0, **how)
    return out + [du, ddelta, dA, dB, dC, dD, dbias] + ([dz] if case["gate"] else []) + ([dh0] if case["state"] else [])


def _own_norm(s):
    import paper_1506_07452_amd as P
    case, x = s["case"], s["x"]
    y = torch.empty_like(x)
    if not case["train"]:
        P.pyramid_group_norm_forward(x, s["gamma"], s["beta"], y, case["G"], act=case["act"], eps=EPS)
        return [y]
    stats = torch.empty((case["N"], case["G"], 2), dtype=torch.float32, device=x.device)
    P.pyramid_group_norm_forward(x, s["gamma"], s["beta"], y, case["G"], act=case["act"], stats=stats, eps=EPS)
    dx = torch.empty_like(x)
    dgamma, dbeta = (torch.empty(case["C"], dtype=torch.float32, device=x.device) for _ in range(2))
    P.pyramid_group_norm_backward(x, s["gamma"], s["beta"], stats, s["dy"], dx, dgamma, dbeta, case["G"], act=case["act"])
    return [y, dx, dgamma, dbeta]


def _own_adamw(s):
    import paper_1506_07452_amd as P
    eight = s["case"]["bits"] == 8
    if "adamw" not in s:
        # the optimiser that a program makes once, here from moments that are there already
        kept = {"m": s["m"], "v": s["v"], "t": s["t"]}
        if eight:
            kept.update(mscale=s["ms"], vscale=s["vs"])
        s["adamw"] = P.AdamW(s["p"], lr=LR, betas=BETAS, eps=ADAM_EPS, weight_decay=DECAY, bits=s["case"]["bits"],
                             copies=s["copies"], state=kept)
    s["adamw"].step(s["g"], grad_scale=s["scale"])
    return [s["p"], s["adamw"].moments(), s["copies"]]


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"conv": _own_conv, "scan": _own_scan, "norm": _own_norm, "adamw": _own_adamw}[kind](state)
    return {"conv": _plain_conv, "scan": _plain_scan, "norm": _plain_norm, "adamw": _plain_adamw}[kind](state)


# ------------------------------------------------------------- the definition, in 64 bits

def _exact_conv(s):
    case = s["case"]
    B, T, I, K = case["B"], case["T"], case["I"], case["K"]
    x, w, bias = (s[k].double().requires_grad_() for k in ("x", "w", "bias"))
    state = s["state"].double() if case["state"] else torch.zeros((B, K - 1, I), dtype=torch.float64, device=x.device)
    state.requires_grad_()
    n = s["lengths"].long() if case["ragged"] else torch.full((B,), T, device=x.device)
    rows = torch.arange(B, device=x.device)[:, None]
    t = torch.arange(T, device=x.device)[None, :]
    s_of = n[:, None] - 1 - t if case["reverse"] else t.expand(B, -1)   # sweep position of a step (below 0 or past n: none)
    has = (t < n[:, None])[:, :, None]
    a = bias.expand(B, T, I)
    for k in range(K):
        p = s_of - (K - 1) + k      # the sweep position that tap k reads
        step = n[:, None] - 1 - p if case["reverse"] else p
        got = torch.where((p >= 0)[:, :, None], x[rows, step.clamp(0, T - 1)], state[rows, (p + K - 1).clamp(0, max(K - 2, 0))])
        a = a + w[:, k] * got
    y = torch.where(has, a / (1 + torch.exp(-a)), torch.zeros_like(a))
    p = n[:, None] - (K - 1) + torch.arange(K - 1, device=x.device)[None, :]
    step = n[:, None] - 1 - p if case["reverse"] else p
    after = torch.where((p >= 0)[:, :, None], x[rows, step.clamp(0, T - 1)], state[rows, (p + K - 1).clamp(0, max(K - 2, 0))])
    out = [y.detach()] + ([after.detach()] if case["state"] else [])
    if not case["train"]:
        return out
    loss = (y * s["dy"].double()).sum()
    if case["state"]:
        loss = loss + (after * s["dstate"].double()).sum()
    dx, dw, db, dstate = torch.autograd.grad(loss, (x, w, bias, state))
    return out + [dx, dw, db] + ([dstate] if case["state"] else [])


def _exact_scan(s):
    case, dev = s["case"], s["u"].device
    B, T, I, S = case["B"], case["T"], case["I"], case["S"]
    rows = torch.arange(B, device=dev)
    n = s["lengths"].long() if case["ragged"] else None

    def at(p):
        # the step at sweep position p (of each sequence, where they differ in length) and where there is one
        if n is None:
            return (T - 1 - p if case["reverse"] else p), None
        return torch.where(p < n, (n - 1 - p) if case["reverse"] else torch.full_like(n, p), torch.full_like(n, p)), p < n

    def take(v, step):
        return v[:, step].double() if n is None else v[rows, step].double()

    def put(v, step, value):
        v[(slice(None) if n is None else rows), step] = value

    def zero(*shape):
        return torch.zeros(shape, dtype=torch.float64, device=dev)

    def mask(has, v):
        return v if has is None else torch.where(has.view(-1, *[1] * (v.dim() - 1)), v, torch.zeros_like(v))

    A, D, dbias = s["A"].double(), s["D"].double(), s["dbias"].double()
    h = s["h0"].double() if case["state"] else zero(B, I, S)
    y, kept = zero(B, T, I), [h]

    def inputs(step, has):
        raw = take(s["delta"], step) + dbias
        dt = mask(has, torch.logaddexp(raw, torch.zeros_like(raw)))
        return mask(has, take(s["u"], step)), raw, dt, mask(has, take(s["B"], step))[:, None], mask(has, take(s["C"], step))[:, None]

    for p in range(T):
        step, has = at(p)
        u, raw, dt, Bt, Ct = inputs(step, has)
        h = (dt[:, :, None] * A).exp() * h + (dt * u)[:, :, None] * Bt
        o = (h * Ct).sum(2) + D * u
        if case["gate"]:
            z = take(s["z"], step)
            o = o * z / (1 + torch.exp(-z))
        put(y, step, mask(has, o))
        if case["train"]:
            kept.append(h)
    out = [y] + ([h] if case["state"] else [])
    if not case["train"]:
        return out
    G = s["dhT"].double() if case["state"] else zero(B, I, S)
    du, ddelta, dz, dB, dC = zero(B, T, I), zero(B, T, I), zero(B, T, I), zero(B, T, S), zero(B, T, S)
    dA, dD, ddb = zero(I, S), zero(I), zero(I)
    for p in range(T - 1, -1, -1):
        step, has = at(p)
        u, raw, dt, Bt, Ct = inputs(step, has)
        h = kept.pop()
        before = kept[-1]
        dp = mask(has, take(s["dy"], step))
        if case["gate"]:
            z = take(s["z"], step)
            sg = 1 / (1 + torch.exp(-z))
            o = (h * Ct).sum(2) + D * u
            put(dz, step, mask(has, dp * o * (sg + z * sg * (1 - sg))))
            dp = mask(has, dp * z * sg)
        put(dC, step, (h * dp[:, :, None]).sum(1))
        G = G + Ct * dp[:, :, None]
        put(dB, step, (G * (dt * u)[:, :, None]).sum(1))
        q = (G * Bt).sum(2)
        put(du, step, dt * q + D * dp)
        G = G * (dt[:, :, None] * A).exp()
        w = G * before
        d = mask(has, (u * q + (w * A).sum(2)) / (1 + torch.exp(-raw)))
        put(ddelta, step, d)
        dA += (w * dt[:, :, None]).sum(0)
        dD += (dp * u).sum(0)
        ddb += d.sum(0)
    return out + [du, ddelta, dA, dB, dC, dD, ddb] + ([dz] if case["gate"] else []) + ([G] if case["state"] else [])


def _exact_norm(s):
    case = s["case"]
    N, V, C, G = case["N"], case["V"], case["C"], case["G"]
    x, gamma, beta = (s[k].double().requires_grad_() for k in ("x", "gamma", "beta"))
    g = x.reshape(N, V, G, C // G)
    var, mean = torch.var_mean(g, dim=(1, 3), unbiased=False, keepdim=True)
    v = ((g - mean) / (var + EPS).sqrt()).reshape(N, V, C) * gamma + beta
    y = v / (1 + torch.exp(-v)) if case["act"] == "silu" else v
    if not case["train"]:
        return [y.detach()]
    return [y.detach()] + list(torch.autograd.grad((y * s["dy"].double()).sum(), (x, gamma, beta)))


def _exact_adamw(s):
    # an update in 64 bits; the moments are fp32 numbers, and 8-bit codes those of them
    case, t, (b1, b2) = s["case"], s["t"] + 1, BETAS
    eight = case["bits"] == 8
    ps, values, copies = [], [], []

    def hashed(x):
        for shift, factor in ((16, 0x7feb352d), (15, 0x846ca68b)):
            x = (x ^ x >> shift) * factor % 2 ** 32
        return x ^ x >> 16

    powers = torch.tensor([2.0 ** e for e in range(-1000, 2)], dtype=torch.float64, device=s["p"][0].device)

    def two(e):
        return powers[e.long() + 1000]

    def value(code, signed):
        k = (code.long() & 127 if signed else code.long()).double()
        e, low = torch.floor(k / 8), -14 if signed else -30
        v = torch.where(e > 0, (1 + (k - 8 * e) / 8) * two((e - 1).clamp(min=0) + low), k / 8 * 2.0 ** low)
        return torch.where(code > 127, -v, v) if signed else v

    def blocks(v):
        return torch.nn.functional.pad(v, (0, -v.numel() % BLOCK)).reshape(-1, BLOCK)

    def coded(x, signed, chance):
        # the codes' values on either side of |x| / scale, the upper one with the probability of how near it is (16 bits of it)
        top = blocks(x.abs()).max(1).values
        r = (blocks(x.abs()) / torch.where(top > 0, top, 1.0)[:, None]).reshape(-1)[:x.numel()]
        e = torch.floor(torch.log2(r.clamp(min=1e-290)))
        e = e - (two(e) > r).double()
        e = torch.clamp(e + (two(e + 1) <= r).double(), min=-14.0 if signed else -30.0)
        grid = two(e - 3)
        low = torch.floor(r / grid)
        up = torch.floor((r / grid - low) * 65536) + chance >= 65536
        k = low + up.double()
        if not signed:
            k = torch.where((r > 0) & (k == 0), torch.ones_like(k), k)
        return (k * grid * top.repeat_interleave(BLOCK)[:x.numel()] * torch.sign(x)).float().double()

    for k, p in enumerate(s["p"]):
        m, v = s["m"][k], s["v"][k]
        if eight:
            m = (blocks(value(m, True)) * s["ms"][k].double()[:, None]).reshape(-1)[:p.numel()].float()
            v = (blocks(value(v, False)) * s["vs"][k].double()[:, None]).reshape(-1)[:p.numel()].float()
        g = s["g"][k].double() * (s["scale"].double() if case["clip"] else 1.0)
        m, v = m.double() * b1 + g * (1 - b1), v.double() * b2 + g * g * (1 - b2)
        m, v, p = m.float().double(), v.float().double(), p.double()
        p = p - LR * (m / (1 - b1 ** t) / ((v / (1 - b2 ** t)).sqrt() + ADAM_EPS) + DECAY * p)
        if eight:
            r = hashed(torch.arange(p.numel(), device=p.device) ^ hashed((hashed(t) + k) % 2 ** 32))
            m, v = coded(m, True, r % 65536), coded(v, False, r // 65536)
        ps.append(p)
        values.append((m, v))
        copies.append(p)
    return [ps, values, copies if s["copies"] is not None else None]


def exact(case, seed):
    s = prepare(case, seed)
    return {"conv": _exact_conv, "scan": _exact_scan, "norm": _exact_norm, "adamw": _exact_adamw}[case["kind"]](s)
