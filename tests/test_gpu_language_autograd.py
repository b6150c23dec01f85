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


def draw_setup():
    """Rows, numbers and settings of a draw, one a row each."""
    gen = torch.Generator().manual_seed(7)
    logits, uniforms = torch.randn(5, 40, generator=gen).to(DEV), torch.rand(5, generator=gen).to(DEV)
    settings = {"temperature": torch.full((5,), 0.7), "top_k": torch.full((5,), 9, dtype=torch.int32),
                "top_p": torch.full((5,), 0.9), "min_p": torch.full((5,), 0.01)}
    return micro.TokenTable(40, 1, 5), logits, uniforms, {k: v.to(DEV) for k, v in settings.items()}


# those of a draw's arguments whose values the logarithms of the shares depend on
DRAWN_FROM = ["logits", "uniforms", "temperature", "top_p", "min_p"]


@pytest.mark.parametrize("given", [False, True], ids=["", "out"])  # the native way, and the other
@pytest.mark.parametrize("name", DRAWN_FROM)
def test_a_draw_from_a_tensor_that_requires_its_gradient(name, given):
    table, logits, uniforms, settings = draw_setup()
    out = torch.full((5,), 7, dtype=torch.int64, device=DEV) if given else None
    want = table.sample(logits, uniforms, **settings)
    args = {"logits": logits, "uniforms": uniforms} | settings
    for made in (lambda t: t.clone().requires_grad_(), torch.nn.Parameter, lambda t: torch.nn.Parameter(t) * 1.0):
        args[name] = made(({"logits": logits, "uniforms": uniforms} | settings)[name])
        with pytest.raises(RuntimeError, match=f"{name} .*no_grad"):
            table.sample(**args, out=out)
        torch.cuda.synchronize()
        assert out is None or bool((out == 7).all())
    with torch.no_grad():
        got = table.sample(**args, out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = table.sample(**(args | {name: args[name].detach()}))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("given", [False, True], ids=["", "out"])
@pytest.mark.parametrize("name", DRAWN_FROM)
def test_a_draw_from_a_tensor_with_a_tangent(name, given):
    table, logits, uniforms, settings = draw_setup()
    out = torch.full((5,), 7, dtype=torch.int64, device=DEV) if given else None
    args = {"logits": logits, "uniforms": uniforms} | settings
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(args[name], torch.ones_like(args[name]))
        with pytest.raises(RuntimeError, match=f"{name} .*tangent"):
            table.sample(**(args | {name: dual}), out=out)
        with torch.no_grad(), pytest.raises(RuntimeError, match="tangent"):
            table.sample(**(args | {name: dual}), out=out)
        torch.cuda.synchronize()
        assert out is None or bool((out == 7).all())
        got = table.sample(**args)  # others of the same level carry none
    want = table.sample(**args)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_packing_and_products_of_tensors_that_carry_a_gradient_or_a_tangent():
    mx = micro.Microscaled()
    x, out = torch.ones(6, 64, device=DEV), torch.full((6, 6), 7.0, device=DEV)
    values = torch.full((6, 64), 7.0, device=DEV)
    q = mx.pack(x)

    def calls(x, out, values):
        return [lambda: mx.pack(x), lambda: mx.pack(x, transposed=True), lambda: mx.pack_both(x), lambda: mx.linear(x, q),
                lambda: mx.linear(x[:1], q), lambda: mx.linear(x, q, out=torch.empty_like(out)),
                lambda: mx.linear(torch.ones(6, 64, device=DEV), q, out=out), lambda: mx.product(q, q, out=out),
                lambda: mx.product(q, q, out=out, accumulate=True), lambda: mx.unpack(q, out=values)]

    for call in calls(x.clone().requires_grad_(), out.requires_grad_(), values.requires_grad_()):
        with pytest.raises(RuntimeError, match="no_grad"):
            call()
    out, values = out.detach(), values.detach()
    with forward_ad.dual_level():
        dual = [forward_ad.make_dual(t, torch.ones_like(t)) for t in (x, out, values)]
        for call in calls(*dual):
            with pytest.raises(RuntimeError, match="tangent"):
                call()
        want = torch.full((6, 6), 64.0, device=DEV)
        assert torch.equal(mx.product(q, q), want) and torch.equal(mx.linear(x, q), want)
    torch.cuda.synchronize()
    assert bool((out == 7).all()) and bool((values == 7).all())
