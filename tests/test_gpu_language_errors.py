"""A call that fails for want of memory leaves nothing behind: the calls after
it, the library's and torch's, succeed."""
import pytest
import torch

import paper_2310_00967_amd as micro
from paper_2310_00967_amd import _lib

pytestmark = pytest.mark.gpu

DEV = "cuda"


def refused_for_memory():
    """The loss's copy of 2^22 hidden rows of 65536 values would take 550 GB."""
    table = micro.TokenTable(8, 65536, 2 ** 22, dtype=torch.bfloat16)
    hidden = torch.zeros(4, 65536, dtype=torch.bfloat16, device=DEV)
    weight = torch.zeros(8, 65536, dtype=torch.bfloat16, device=DEV)
    targets = torch.zeros(4, dtype=torch.int64, device=DEV)
    with pytest.raises(_lib.MicroError) as e:
        table.loss(hidden, weight, targets)
    assert e.value.status == _lib.MICRO_ENOMEM and "scratch" in str(e.value)


def test_the_next_calls_succeed():
    weight = torch.arange(40.0, device=DEV).view(5, 8)
    ids = torch.tensor([3, 0, 3], device=DEV)
    table = micro.TokenTable(5, 8, 4)
    small = [torch.ones(100, device=DEV)]
    grads = micro.GradientSet(small)
    torch.cuda.synchronize()
    refused_for_memory()
    rows = table.lookup(weight, ids)
    refused_for_memory()
    dweight = table.lookup_grad(rows, ids, torch.empty(5, 8, device=DEV))
    refused_for_memory()
    norm = grads.norm()
    refused_for_memory()
    loss, losses = table.loss(rows, weight, ids)
    refused_for_memory()
    twice = weight * 2
    torch.cuda.synchronize()
    assert torch.equal(rows, weight[ids]) and torch.equal(dweight[3], 2 * weight[3])
    assert float(norm) == 10.0 and bool(losses.isfinite().all()) and torch.equal(twice, weight + weight)
    refused_for_memory()
    sp = micro.Sparsifier(1000)
    residual = torch.zeros(1000, device=DEV)
    refused_for_memory()
    k, _, idx, val = sp.step(torch.ones(1000, device=DEV), residual, 0, 1, 0.1, 0.5)
    assert k == 1000
