"""Edges of the block operators on the GPU: tensors that are given other memory between updates, more work than a
launch takes, arguments that are left out, numbers at the ends of fp32, and sums that are held in 64 bits."""
from __future__ import annotations

import pytest
import torch

import paper_1506_07452_amd as P
from tests.gpu_util import DEV, say
from tests.test_gpu_sequence import BF16, F32, rand

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
