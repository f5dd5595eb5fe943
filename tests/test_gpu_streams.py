"""Calls given another stream than the current one, which is still busy when they
return: no memory that they drop is handed to the current stream's next tensors."""
from __future__ import annotations

import pytest
import torch

import paper_1506_07452_amd as P
from paper_1506_07452_amd import network as net
from tests.gpu_util import DEV, say
from tests.test_gpu_network_norm import case

pytestmark = pytest.mark.gpu

NAN = float("nan")


def idle_blocks():
    """Sizes of the blocks that the current stream's next tensors may get."""
    mine = torch.cuda.current_stream().cuda_stream
    return [b["size"] for seg in torch.cuda.memory_snapshot() if seg["stream"] == mine
            for b in seg["blocks"] if b["state"] == "inactive"]


def beside_busy_stream(call, as_handle=False):
    """call(stream)'s result, the stream having work before it; all the memory that
    the current stream can give away after the call is filled with NaN."""
    side = torch.cuda.Stream()
    a = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(side):
        out = a @ a
    call(side)                      # the stream has its memory: the next call waits for none
    torch.cuda.synchronize()
    before = sum(idle_blocks())
    with torch.cuda.stream(side):
        for _ in range(150):
            out = a @ a
    out = call(side.cuda_stream if as_handle else side)
    idle = idle_blocks()
    junk = [torch.full((n // 4,), NAN, device=DEV) for n in idle]
    torch.cuda.synchronize()
    del junk
    # the call itself may not have dropped anything there
    assert sum(idle) <= before
    return out


def same(got, want):
    a, b = list(net._tensors(got)), list(net._tensors(want))
    assert len(a) == len(b) > 0
    for u, v in zip(a, b):
        if u.dtype == torch.uint8:      # saved buffers: the gaps between their arrays hold anything
            continue
        assert torch.equal(u, v)


@pytest.mark.parametrize("raw", [False, True], ids=["stream", "handle"])
@pytest.mark.parametrize("own_ws", [False, True], ids=["ws", "no-ws"])
@pytest.mark.parametrize("eight", [False, True], ids=["plain", "checkpoint8"])
@pytest.mark.parametrize("last_fc,fused", [(True, True), (True, False), (False, True)])
def test_training_step(last_fc, fused, eight, own_ws, raw):
    d, _ = case([16, 32, 16], last_fc, 51, (1, 0, 1))
    ws = None if own_ws else net.workspace_for(d["x"].shape, [16, 32, 16], True, torch.float32, True, DEV)
    args = (d["x"], d["layers"], d["fcs"], d["head"], d["labels"])
    kw = dict(ws=ws, fused_head=fused, norms=d["norms"], checkpoint8=eight)
    want = net.network_train_step(*args, **kw)
    say("training step beside a busy stream", last_fc, fused, eight, own_ws, raw)
    same(beside_busy_stream(lambda s: net.network_train_step(*args, stream=s, **kw), raw), want)


@pytest.mark.parametrize("normed", [(0, 0, 0), (1, 1, 1)])
def test_inference_and_volumes(normed):
    d, _ = case([16, 32, 16], True, 52, normed)
    args = (d["x"], d["layers"], d["fcs"], d["head"])
    ws = net.workspace_for(d["x"].shape, [16, 32, 16], True, torch.float32, False, DEV)
    say("inference beside a busy stream", normed)
    want = net.network_forward(*args, norms=d["norms"], ws=ws)["p"]
    # the stream by position
    got = beside_busy_stream(lambda s: net.network_forward(*args, None, False, ws, s, norms=d["norms"])["p"])
    same(got, want)
    volume = dict(tile=(3, 6, 7), stride=(1, 3, 4), norms=d["norms"], ws=ws)
    want = net.network_infer_volume(*args, **volume)
    same(beside_busy_stream(lambda s: net.network_infer_volume(*args, stream=s, **volume)), want)


def test_results_are_the_callers_too():
    """A result that the caller's stream still reads when it is dropped is not given
    to the call's stream in the meantime."""
    d, _ = case([16, 32], True, 53, (1, 1))
    args = (d["x"], d["layers"], d["fcs"], d["head"], d["labels"])
    side = torch.cuda.Stream()
    want = net.network_train_step(*args, norms=d["norms"])["p"].clone()
    a = torch.randn(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    out = net.network_train_step(*args, stream=side, norms=d["norms"])
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(40):
        a @ a
    got = out["p"] * 1.0
    size = out["p"].numel()
    del out
    with torch.cuda.stream(side):
        junk = [torch.full((size,), NAN, device=DEV) for _ in range(8)]
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    del junk


def entry_points():
    """name: (call(stream) on tensors made here, its outputs)."""
    gen = torch.Generator().manual_seed(54)

    def rand(*shape):
        return (torch.randn(shape, generator=gen) * 0.2).to(DEV)

    def empty(*like):
        return [torch.empty_like(t) for t in like]

    out = {}
    # channels and units of the plane steps, whose workspace is large
    x, h, dh = rand(1, 6, 24, 25, 20), rand(1, 6, 24, 25, 32), rand(1, 6, 24, 25, 32)
    wx, wh, b = rand(6, 128, 20, 3, 3), rand(6, 128, 32, 3, 3), rand(6, 128)
    s = P.shape_for(x, 32)
    saved = torch.empty(P.pyramid_lstm_saved_size(s), dtype=torch.uint8, device=DEV)
    P.pyramid_lstm_forward(s, x, wx, wh, b, h, saved)
    h1, g1 = torch.empty_like(h), empty(x, wx, wh, b)
    out["lstm_forward"] = (lambda st: P.pyramid_lstm_forward(s, x, wx, wh, b, h1, stream=st), [h1])
    out["lstm_backward"] = (lambda st: P.pyramid_lstm_backward(s, x, wx, wh, b, saved, dh, *g1, stream=st), g1)
    x2, h2, dh2 = rand(2, 24, 25, 20), rand(2, 24, 25, 32), rand(2, 24, 25, 32)
    wx2, wh2, b2 = rand(4, 128, 20, 3), rand(4, 128, 32, 3), rand(4, 128)
    s2 = P.shape2d_for(x2, 32)
    saved2 = torch.empty(P.pyramid_lstm2d_saved_size(s2), dtype=torch.uint8, device=DEV)
    P.pyramid_lstm2d_forward(s2, x2, wx2, wh2, b2, h2, saved2)
    h3, g3 = torch.empty_like(h2), empty(x2, wx2, wh2, b2)
    out["lstm2d_forward"] = (lambda st: P.pyramid_lstm2d_forward(s2, x2, wx2, wh2, b2, h3, stream=st), [h3])
    out["lstm2d_backward"] = (
        lambda st: P.pyramid_lstm2d_backward(s2, x2, wx2, wh2, b2, saved2, dh2, *g3, stream=st), g3)
    M = 5000
    rows, w, bias, dy = rand(M, 32), rand(64, 32), rand(64), rand(M, 64)
    y = torch.empty_like(dy)
    P.pyramid_fc_tanh_forward(rows, w, bias, y)
    g4 = empty(rows, w, bias)
    out["fc_backward"] = (lambda st: P.pyramid_fc_tanh_backward(rows, w, y, dy, *g4, stream=st), g4)
    labels = torch.randint(0, 4, (M,), generator=gen, dtype=torch.int32).to(DEV)
    hw, hb = rand(4, 32), rand(4)
    for squared in (False, True):
        g5 = [torch.empty((M, 4), device=DEV), torch.empty(1, device=DEV)] + empty(rows, hw, hb)

        def softmax(st, g=g5, sq=squared):
            P.pyramid_softmax_ce(rows, hw, hb, g[0], labels, *g[1:], stream=st, squared=sq)
        out["softmax_sq" if squared else "softmax_ce"] = (softmax, g5)
    hw2 = rand(4, 64)
    g6 = [torch.empty((M, 4), device=DEV), torch.empty(1, device=DEV)] + empty(rows, w, bias, hw2, hb)
    out["head_train"] = (lambda st: P.pyramid_head_train(rows, w, bias, hw2, hb, labels, *g6, stream=st), g6)
    return out


@pytest.mark.parametrize("raw", [False, True], ids=["stream", "handle"])
@pytest.mark.parametrize("name", ["lstm_forward", "lstm_backward", "lstm2d_forward", "lstm2d_backward", "fc_backward",
                                  "softmax_ce", "softmax_sq", "head_train"])
def test_workspace_made_by_the_binding(name, raw):
    call, outs = entry_points()[name]
    say("workspace of", name, raw)
    call(None)
    want = [t.clone() for t in outs]
    for t in outs:
        t.fill_(NAN)
    beside_busy_stream(call, raw)
    same(outs, want)


@pytest.mark.parametrize("eight", [False, True], ids=["plain", "checkpoint8"])
def test_training_step_captured_on_a_forked_stream(eight):
    """A graph whose step runs on a stream forked from the captured one, replayed with other
    work between the replays."""
    d, _ = case([16, 32, 16], True, 55, (1, 0, 1))
    args = (d["layers"], d["fcs"], d["head"], d["labels"])
    x = d["x"].clone()
    kw = dict(norms=d["norms"], checkpoint8=eight)
    want = net.network_train_step(x, *args, **kw)
    other = x * 0.5
    want_other = net.network_train_step(other, *args, **kw)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    say("captured step", eight)
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = net.network_train_step(x, *args, stream=side, **kw)
        torch.cuda.current_stream().wait_stream(side)
    first = x.clone()
    for turn in range(3):
        for v, w in ((first, want), (other, want_other)):
            x.copy_(v)
            graph.replay()
            net.network_train_step(other, *args, **kw)
            torch.cuda.synchronize()
            same(got, w)
