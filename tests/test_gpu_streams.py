"""Calls given another stream than the current one, which is still busy when they
return: no memory that they drop is handed to the current stream's next tensors."""
from __future__ import annotations

import pytest
import torch

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
