"""Edges of the block operators on the GPU: tensors that are given other memory between updates, more work than a
launch takes, arguments that are left out, numbers at the ends of fp32, and sums that are held in 64 bits."""
from __future__ import annotations

import pytest
import torch

import paper_1506_07452_amd as P
from tests import block_ref as R
from tests.gpu_util import DEV, say
from tests.seq_ref import rounded
from tests.test_gpu_block import gn_case
from tests.test_gpu_sequence import BF16, F32, near, rand

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
