"""The token table's calls are outside autograd: a result that a graph would have
to hold is refused instead of being returned without one."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

import paper_2310_00967_amd as micro

pytestmark = pytest.mark.gpu

DEV = "cuda"


def setup():
    gen = torch.Generator().manual_seed(2)
    weight = torch.randn(30, 16, generator=gen).to(DEV)
    hidden = torch.randn(9, 16, generator=gen).to(DEV)
    ids = torch.randint(0, 30, (9,), generator=gen).to(DEV)
    return micro.TokenTable(30, 16, 9), weight, hidden, ids


def calls(table, weight, hidden, ids, out, dweight):
    return [lambda: table.lookup(weight, ids), lambda: table.lookup(weight, ids, out=out),
            lambda: table.lookup_grad(hidden, ids, dweight), lambda: table.loss(hidden, weight, ids),
            lambda: table.loss_grad(hidden, weight, ids, dhidden=out, dweight=dweight)]


def test_a_tensor_that_requires_its_gradient():
    table, weight, hidden, ids = setup()
    out, dweight = torch.full((9, 16), 7.0, device=DEV), torch.full((30, 16), 7.0, device=DEV)
    want = table.lookup(weight, ids), table.loss(hidden, weight, ids)
    wp, hp = torch.nn.Parameter(weight.clone()), hidden.clone().requires_grad_()
    for i, call in enumerate(calls(table, wp, hp, ids, out, dweight)):
        with pytest.raises(RuntimeError, match="no_grad"):
            call()
    with pytest.raises(RuntimeError, match="no_grad"):  # a tensor of a graph
        table.lookup(wp * 2.0, ids)
    with pytest.raises(RuntimeError, match="no_grad"):  # an output
        table.lookup_grad(hidden, ids, wp)
    torch.cuda.synchronize()
    assert bool((out == 7).all()) and bool((dweight == 7).all()) and torch.equal(wp, weight)
    with torch.no_grad():
        assert torch.equal(table.lookup(wp, ids), want[0])
        assert torch.equal(table.loss(hp, wp, ids)[1], want[1][1])
        for call in calls(table, wp, hp, ids, out, dweight):
            call()
    assert torch.equal(table.lookup(wp.detach(), ids), want[0])


def test_a_tensor_with_a_tangent():
    table, weight, hidden, ids = setup()
    out, dweight = torch.full((9, 16), 7.0, device=DEV), torch.full((30, 16), 7.0, device=DEV)
    with forward_ad.dual_level():
        w = forward_ad.make_dual(weight, torch.ones_like(weight))
        h = forward_ad.make_dual(hidden, torch.ones_like(hidden))
        for call in calls(table, w, h, ids, out, dweight):
            with pytest.raises(RuntimeError, match="tangent"):
                call()
        assert torch.equal(table.lookup(weight, ids), weight[ids])
    torch.cuda.synchronize()
    assert bool((out == 7).all()) and bool((dweight == 7).all())
