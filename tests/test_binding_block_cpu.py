"""What the binding of the block operators passes on and refuses, on the CPU: the questions that need a device
are answered by stand-ins, calls are recorded and not made."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_1506_07452_amd as P

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    """Host tensors stand for a device's; calls of entry points end up in the list."""
    made = []

    def main(name, t, dims):
        assert t.is_contiguous()
        return P._DT[t.dtype], t.data_ptr(), 0

    def tensor(name, t, shape, dtype, dev):
        if t is None:
            return None
        if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
            raise ValueError(name)
        return t.data_ptr()

    def run(name, dev, stream, *args):
        row = {"name": name, "args": args}
        if name.startswith("pyramid_adamw"):
            row["segs"] = [{f: getattr(s, f) for f, _ in P.plstm_adamw_segment._fields_} for s in args[1]]
        made.append(row)

    monkeypatch.setattr(P, "_main", main)
    monkeypatch.setattr(P, "_tensor", tensor)
    monkeypatch.setattr(P, "_run", run)
    return made


SIZES = (300, 17, 256)


def optimiser(bits=8, copies=True, **kw):
    params = [torch.zeros(n) for n in SIZES]
    return P.AdamW(params, bits=bits, copies=[torch.zeros(n, dtype=BF16) if k != 1 else None for k, n in enumerate(SIZES)] if copies else None,
                   **kw), [torch.ones(n) for n in SIZES]


def addresses(opt):
    """What an update has to work on: the tensors that the optimiser shows."""
    rows = []
    for k, p in enumerate(opt.params):
        row = dict(theta=p, m=opt.m[k], v=opt.v[k])
        if opt.bits == 8:
            row.update(mscale=opt.mscale[k], vscale=opt.vscale[k])
        if opt.copies is not None and opt.copies[k] is not None:
            row["copy"] = opt.copies[k]
        rows.append({f: t.data_ptr() for f, t in row.items()})
    return rows


def follows(opt, grads, calls):
    calls.clear()
    opt.step(grads)
    for row, seg in zip(addresses(opt), calls[0]["segs"]):
        assert {f: seg[f] for f in row} == row


@pytest.mark.parametrize("bits", [32, 8])
def test_update_follows_its_tensors(bits, calls):
    """An update works on the parameters and copies that are there now, whichever of them was given other memory or replaced."""
    opt, grads = optimiser(bits)
    follows(opt, grads, calls)
    held = []           # the memory of before stays taken: other memory has other addresses
    for tensors in (opt.params, opt.copies):
        held.append(tensors[0].data)
        tensors[0].data = tensors[0].data.clone()
        follows(opt, grads, calls)
        held.append(tensors[2])
        tensors[2] = tensors[2].clone()
        follows(opt, grads, calls)
    opt.copies[1] = torch.zeros(17, dtype=BF16)
    follows(opt, grads, calls)
    opt.copies[0] = None
    follows(opt, grads, calls)
    assert calls[0]["segs"][0]["copy"] is None
    # what does not fit is refused
    t = opt.t
    for tensors in (opt.params, opt.copies):
        kept = tensors[2]
        tensors[2] = torch.zeros(5, dtype=kept.dtype)
        with pytest.raises(ValueError):
            opt.step(grads)
        tensors[2] = kept
    assert opt.t == t
    follows(opt, grads, calls)


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
def test_moments_stay_where_they_are(bits, given, calls):
    """The moments' memory is held by the optimiser: tensors that show it, the caller's own among them, can be given
    other memory, and lists changed, without the update's going anywhere else."""
    opt, grads = optimiser(bits, copies=False)
    names = ["m", "v"] + (["mscale", "vscale"] if bits == 8 else [])
    state = opt.state()
    if given:
        opt = P.AdamW(opt.params, bits=bits, state=state)
    before = addresses(opt)
    for name in names:
        held = state[name][0].data
        state[name][0].data = torch.zeros_like(held)        # a shown tensor, or the one that was given
        state[name][1] = torch.zeros_like(state[name][1])
        getattr(opt, name)[0].data = torch.zeros_like(held)
        with pytest.raises(AttributeError):
            setattr(opt, name, list(getattr(opt, name)))
        with pytest.raises(TypeError):
            getattr(opt, name)[0] = torch.zeros_like(held)
    follows(opt, grads, calls)
    assert addresses(opt) == before
    for name in names:
        getattr(opt, name)[1].fill_(3)
        assert (opt.state()[name][1] == 3).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_updated_memory_is_apart(bits, calls):
    """What an update writes is refused where two of its tensors share memory, in part or whole."""
    moment = dict(dtype=F32 if bits == 32 else torch.uint8)
    whole, rest = torch.zeros(600), torch.zeros(200)
    codes = torch.zeros(2048, **moment)
    halves = torch.zeros(600, dtype=BF16)
    scales = torch.zeros(8)

    def make(params=(whole[:300], whole[300:]), m=(codes[:300], codes[512:812]), v=(codes[1024:1324], codes[1536:1836]),
             copies=(halves[:300], halves[300:]), ms=(scales[:2], scales[2:4]), vs=(scales[4:6], scales[6:])):
        state = dict(m=list(m), v=list(v), t=3, mscale=list(ms), vscale=list(vs))
        return P.AdamW(params, bits=bits, state=state, copies=copies)

    opt = make()                # neighbours touch
    opt.step([rest.new_ones(300)] * 2)
    for bad in (dict(params=(whole[:300], whole[299:599])), dict(params=(whole[:300], whole[:300])), dict(params=(whole[:300], whole[100:400])),
                dict(m=(codes[:300], codes[299:599])), dict(v=(codes[1024:1324], codes[200:500])), dict(copies=(halves[:300], halves[200:500])),
                dict(copies=(halves[:300], halves[:300])), dict(copies=(halves[:300], whole.view(BF16)[900:1200]))):
        with pytest.raises(ValueError):
            make(**bad)
    if bits == 8:
        for bad in (dict(ms=(scales[:2], scales[1:3])), dict(vs=(scales[1:3], scales[6:])), dict(vs=(scales[4:6], scales[5:7]))):
            with pytest.raises(ValueError):
                make(**bad)
    # also where memory comes to overlap later
    opt.copies[1].data = halves[299:599]
    with pytest.raises(ValueError):
        opt.step([rest.new_ones(300)] * 2)
    one = dict(m=[codes[:200]], v=[codes[512:712]], mscale=[scales[:1]], vscale=[scales[1:2]])
    if bits == 8:
        calls.clear()
        P.pyramid_adamw_moments(**one, mout=[rest], vout=[torch.zeros(200)])
        assert len(calls) == 1
        for out in (dict(mout=[rest], vout=[rest]), dict(mout=[whole[:200]], vout=[whole[100:300]]), dict(mout=[rest], vout=[])):
            with pytest.raises(ValueError):
                P.pyramid_adamw_moments(**one, **out)
        assert len(calls) == 1
    with pytest.raises(ValueError):
        P.pyramid_adamw_step([whole[:300], whole[200:500]], [whole.new_ones(300)] * 2, [codes[:300], codes[512:812]],
                             [codes[1024:1324], codes[1536:1836]], 1e-3, 1, mscale=[scales[:2], scales[2:4]],
                             vscale=[scales[4:6], scales[6:]])


# a tensor's attributes, not a tensor's type
FOREIGN = [np.zeros((2, 4), np.float32), [0.0], "ab", 3]


@pytest.mark.parametrize("t", FOREIGN, ids=lambda t: type(t).__name__)
def test_arrays_of_others(t, monkeypatch):
    """Where a tensor is expected anything else is a TypeError, as for main tensors."""
    with pytest.raises(TypeError):
        P._tensor("t", t, (2, 4), F32, 0)
    with pytest.raises(TypeError):
        P._pitched("t", t, (1, 2, 4), F32, 0)
    x, w = torch.zeros((1, 2, 4)), torch.zeros((4, 4))
    monkeypatch.setattr(P, "_main_pitched", lambda name, t: (0, -1, t.data_ptr(), 0))
    monkeypatch.setattr(P, "_main", lambda name, t, dims: (0, t.data_ptr(), -1))
    monkeypatch.setattr(P, "_run", lambda *a: pytest.fail("called"))
    for other in (t, None):
        with pytest.raises(TypeError):
            P.pyramid_causal_conv_forward(x, other, None, x)
        with pytest.raises(TypeError):
            P.pyramid_causal_conv_backward(x, other, None, x, x, w, None, ws=x)
        with pytest.raises(TypeError):
            P.pyramid_selective_scan_forward(x, x, other, x, x, x, ws=x)
    with pytest.raises(TypeError):
        P.pyramid_causal_conv_forward(x, w, t, x)
    with pytest.raises(TypeError):
        P.pyramid_selective_scan_forward(x, t, w, x, x, x, ws=x)
    p = [torch.zeros(4), torch.zeros(4)]
    opt = P.AdamW(p)
    for grads in ([t, t], [torch.ones(4), t]):
        with pytest.raises(TypeError):
            opt.step(grads)
    with pytest.raises(TypeError):
        P.pyramid_adamw_step(p, [None, None], [t, t], p, 1e-3, 1)
    with pytest.raises(TypeError):
        P.AdamW(p, copies=[t, None])
