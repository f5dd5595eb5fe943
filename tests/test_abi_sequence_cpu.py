"""Refusals of the layer norm, scan and checkpoint entry points (C ABI, no GPU:
validation comes before any HIP call), and the 64-bit forms that the GPU tests
use, against autograd and differences."""
from __future__ import annotations

import ctypes

import pytest
import torch

import paper_1506_07452_amd as P
from tests import seq_ref as R

FAKE = ctypes.c_void_p(0x10000)      # aligned, never dereferenced
ODD = ctypes.c_void_p(0x10001)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return P.load()


def norm_fwd(lib, M=4, C=8, dtype=0, eps=1e-5, x=FAKE, gamma=FAKE, beta=FAKE, y=FAKE, stats=None, xq=None, xscale=None):
    return lib.pyramid_layer_norm_forward(M, C, dtype, eps, x, gamma, beta, y, stats, xq, xscale, None)


def norm_bwd(lib, M=4, C=8, dtype=0, x=FAKE, xscale=None, gamma=FAKE, stats=FAKE, dy=FAKE, dx=FAKE, dgamma=FAKE,
             dbeta=FAKE, ws=FAKE, nbytes=0):
    return lib.pyramid_layer_norm_backward(M, C, dtype, x, xscale, gamma, stats, dy, dx, dgamma, dbeta, ws, nbytes, None)


def test_norm_refusals(lib):
    for bad in (dict(M=0), dict(M=-1), dict(C=0), dict(dtype=2), dict(dtype=-1), dict(eps=0.0), dict(eps=-1.0),
                dict(eps=float("nan")), dict(x=None), dict(gamma=None), dict(beta=None), dict(y=None), dict(x=ODD),
                dict(y=ODD), dict(stats=ODD), dict(xq=FAKE), dict(xscale=FAKE), dict(xq=ODD, xscale=FAKE)):
        assert norm_fwd(lib, **bad) == -1, bad
    for bad in (dict(C=16385), dict(M=(1 << 32) + 1), dict(M=1 << 31, C=1024)):
        assert norm_fwd(lib, **bad) == -2, bad
    for bad in (dict(M=0), dict(C=0), dict(dtype=9), dict(x=None), dict(gamma=None), dict(stats=None), dict(dy=None),
                dict(dgamma=None), dict(dbeta=None), dict(ws=None), dict(dx=ODD), dict(xscale=ODD), dict(ws=ODD)):
        assert norm_bwd(lib, nbytes=BIG, **bad) == -1, bad
    assert norm_bwd(lib, C=20000, nbytes=BIG) == -2
    need = P.pyramid_layer_norm_workspace_size(4, 8)
    assert need > 0 and norm_bwd(lib, nbytes=need - 1) == -3
    for bad in ((0, 8), (4, 0), (4, 20000), (1 << 40, 8)):
        assert P.pyramid_layer_norm_workspace_size(*bad) == 0


def scan_fwd(lib, B=2, T=5, I=8, dtype=0, reverse=0, g=FAKE, u=FAKE, lengths=None, h0=None, h=FAKE, hT=None, saved=None,
             ws=FAKE, nbytes=BIG):
    return lib.pyramid_scan_forward(B, T, I, dtype, reverse, g, u, lengths, h0, h, hT, saved, ws, nbytes, None)


def scan_bwd(lib, B=2, T=5, I=8, dtype=0, reverse=0, g=FAKE, gscale=None, u=FAKE, uscale=None, lengths=None, saved=FAKE,
             dh=FAKE, dhT=None, dg=FAKE, du=FAKE, dh0=None, ws=FAKE, nbytes=BIG):
    return lib.pyramid_scan_backward(B, T, I, dtype, reverse, g, gscale, u, uscale, lengths, saved, dh, dhT, dg, du, dh0,
                                     ws, nbytes, None)


def test_scan_refusals(lib):
    for bad in (dict(B=0), dict(T=0), dict(I=0), dict(T=-3), dict(dtype=2), dict(reverse=2), dict(reverse=-1), dict(g=None),
                dict(u=None), dict(h=None), dict(ws=None), dict(g=ODD), dict(h0=ODD), dict(hT=ODD), dict(saved=ODD),
                dict(lengths=ODD), dict(ws=ODD)):
        assert scan_fwd(lib, **bad) == -1, bad
    for bad in (dict(T=(1 << 31) + 1), dict(B=1 << 20, T=1 << 20), dict(B=1 << 30, I=1 << 30), dict(I=1 << 62)):
        assert scan_fwd(lib, **bad) == -2, bad
    assert scan_fwd(lib, nbytes=P.pyramid_scan_workspace_size(2, 5, 8) - 1) == -3
    for bad in (dict(B=0), dict(dtype=5), dict(reverse=3), dict(g=None), dict(u=None), dict(saved=None), dict(dh=None),
                dict(dg=None), dict(du=None), dict(ws=None), dict(gscale=FAKE), dict(uscale=FAKE), dict(dg=ODD), dict(dhT=ODD),
                dict(dh0=ODD)):
        assert scan_bwd(lib, **bad) == -1, bad
    assert scan_bwd(lib, T=1 << 40) == -2
    assert scan_bwd(lib, nbytes=0) == -3
    for bad in ((0, 5, 8), (2, 0, 8), (2, 5, -1), (1 << 20, 1 << 20, 1)):
        assert P.pyramid_scan_workspace_size(*bad) == 0 and P.pyramid_scan_saved_size(*bad) == 0
    assert P.pyramid_scan_saved_size(2, 33, 8) >= 2 * 3 * 8 * 4


def test_checkpoint_refusals(lib):
    for fn, args in ((lib.pyramid_checkpoint8_pack, 3), (lib.pyramid_checkpoint8_unpack, 3)):
        assert fn(0, 0, FAKE, FAKE, FAKE, None) == -1
        assert fn(-5, 0, FAKE, FAKE, FAKE, None) == -1
        assert fn(5, 2, FAKE, FAKE, FAKE, None) == -1
        assert fn(1 << 39, 0, FAKE, FAKE, FAKE, None) == -2
        for k in range(args):
            for v in (None, ODD):
                p = [FAKE] * args
                p[k] = v
                assert fn(5, 0, *p, None) == -1
    assert [P.pyramid_checkpoint8_scales(n) for n in (-1, 0, 1, 64, 65)] == [0, 0, 1, 1, 2]


def test_binding_refuses_host_tensors():
    x, v = torch.zeros((4, 8)), torch.zeros(8)
    with pytest.raises(ValueError):
        P.pyramid_layer_norm_forward(x, v, v, x)
    with pytest.raises(ValueError):
        P.pyramid_scan_forward(x[None], x[None], x[None])
    with pytest.raises(ValueError):
        P.pyramid_checkpoint8_pack(x, *P.checkpoint8_empty(x))
    with pytest.raises(TypeError):
        P.pyramid_layer_norm_forward(None, v, v, x)


def test_norm_forms_against_autograd():
    gen = torch.Generator().manual_seed(1)
    x, dy = (torch.randn((9, 13), generator=gen, dtype=torch.float64) for _ in range(2))
    w, b = (torch.randn(13, generator=gen, dtype=torch.float64) for _ in range(2))
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    y = torch.nn.functional.layer_norm(leaves[0], (13,), leaves[1], leaves[2], 1e-5)
    y.backward(dy)
    ry, _, mean, rstd = R.norm_forward(x, w, b, 1e-5, torch.float32)
    got = [ry] + [v for v, _ in R.norm_backward(x, mean, rstd, w, dy, torch.float32)]
    for a, want in zip(got, [y.detach()] + [t.grad for t in leaves]):
        assert (a - want).abs().max() <= 1e-12 * (1 + want.abs().max())


@pytest.mark.parametrize("reverse", [False, True])
def test_scan_forms_against_autograd(reverse):
    gen = torch.Generator().manual_seed(2)
    B, T, I, lengths = 3, 19, 2, [19, 0, 7]
    g, u, dh = (torch.randn((B, T, I), generator=gen, dtype=torch.float64) for _ in range(3))
    h0, dhT = (torch.randn((B, I), generator=gen, dtype=torch.float64) for _ in range(2))
    leaves = [t.clone().requires_grad_() for t in (g, u, h0)]
    loss = 0
    for b, n in enumerate(lengths):
        v = leaves[2][b]
        for s in range(n):
            t = n - 1 - s if reverse else s
            f = 1 / (1 + torch.exp(-leaves[0][b, t]))
            v = f * v + (1 - f) * leaves[1][b, t]
            loss = loss + (v * dh[b, t]).sum()
        loss = loss + (v * dhT[b]).sum()
    loss.backward()
    h, _, hT, _, before, eb = R.scan_forward(g, u, reverse, lengths, h0)
    assert torch.equal(hT[1], h0[1]) and not h[1].any()
    got = [v for v, _ in R.scan_backward(g, u, before, eb, dh, reverse, lengths, dhT)]
    for a, leaf in zip(got, leaves):
        assert (a - leaf.grad).abs().max() <= 1e-12


def test_code_forms():
    """Every value within half a scale, the scale the smallest bf16 that
    serves, the codes of a block within 127."""
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(640, generator=gen) * torch.exp2(torch.arange(640) / 10 - 32)
    q, s, v = R.codes(x)
    blocks = x.double().view(-1, 64)
    top = blocks.abs().amax(1)
    sd = s.double()
    assert (sd * 127 >= top).all() and (sd * 127 <= top * (1 + 2.0 ** -7) * (1 + 1e-12)).all()
    below = (s.view(torch.int16) - 1).view(torch.bfloat16).double()
    assert (below * 127 < top).all()
    assert ((v.view(-1, 64) - blocks).abs() <= sd[:, None] / 2).all()
    assert q.abs().max() <= 127


def test_saved_buffers_of_another_shape_are_refused():
    """The arrays that 8-bit checkpoints pack cover a saved buffer of their shape exactly."""
    from paper_1506_07452_amd import network as net
    for N, D, H, W, C, O, K in ((1, 3, 4, 5, 2, 16, 3), (2, 1, 1, 1, 1, 4, 1), (1, 5, 7, 3, 9, 32, 5)):
        s = P.plstm_shape(N, D, H, W, C, O, 0, K)
        size = P.pyramid_lstm_saved_size(s)
        arrays = net._saved_arrays(torch.empty(size, dtype=torch.uint8), s)
        cells = 6 * N * D * H * W * O
        assert [a.numel() for a in arrays] == [4 * cells, cells, cells]
        for bad in (size - 4, size + 256, size // 2):
            with pytest.raises(ValueError):
                net._saved_arrays(torch.empty(bad, dtype=torch.uint8), s)
