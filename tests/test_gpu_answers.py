"""The 4-bit products and the draw together with the token table's other calls, as a
program uses them: a layer trained through packed products between lookup and loss, and
a model's answers."""
import os
import sys

import pytest
import torch

import paper_2310_00967_amd as micro

import language_reference
import microscaled_reference as ref
import sample_reference

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import tied_language_model as example  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda"


def test_a_layer_between_lookup_and_loss():
    """Every call's output against its definition on the inputs that it got."""
    vocab, dim, out, tokens = 900, 96, 160, 333
    gen = torch.Generator().manual_seed(4)
    weight = torch.randn(vocab, dim, generator=gen).to(DEV)
    layer = torch.randn(out, dim, generator=gen).mul_(0.1).to(DEV)
    head = torch.randn(vocab, out, generator=gen).mul_(0.1).to(DEV)
    x, y = (torch.randint(0, vocab, (tokens,), generator=gen).to(DEV) for _ in range(2))
    table, loss_table = micro.TokenTable(vocab, dim, tokens), micro.TokenTable(vocab, out, tokens)
    mx = micro.Microscaled()
    rows = table.lookup(weight, x)
    q, qt = mx.pack_both(rows)
    w, wt = mx.pack_both(layer)
    hidden = mx.product(q, w)
    _, _, dhidden, dhead = loss_table.loss_grad(hidden, head, y)
    d, dt = mx.pack_both(dhidden)
    drows = mx.product(d, wt)
    dlayer = mx.product(dt, qt)
    dweight = table.lookup_grad(drows, x, torch.zeros_like(weight))
    grads = micro.GradientSet([dweight, dlayer, dhead])
    flat = torch.empty(grads.n_total, device=DEV)
    norm = grads.flatten(flat, max_norm=1e9)
    v = lambda t: ref.packed_values(t.cpu())  # noqa: E731
    for got, a, b in ((hidden, rows, layer), (drows, dhidden, layer.t()), (dlayer, dhidden.t(), rows.t())):
        want, bound = ref.product(v(a), v(b), torch.float32)
        assert language_reference.excess(got, want, bound) <= 1.0
    want, bound = language_reference.lookup_grad(drows.cpu(), x.cpu(), vocab, 1.0, None)
    assert language_reference.excess(dweight, want, bound) <= 1.0
    parts = flat.split([t.numel() for t in (dweight, dlayer, dhead)])
    assert torch.equal(parts[1], dlayer.flatten()) and float(norm) > 0
    # captured and replayed with other values, beside the eager calls
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    on = micro.Microscaled(stream=stream)
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            gq, gqt = on.pack_both(rows)
            gw, _ = on.pack_both(layer)
            gy = on.product(gq, gw)
            gd = on.product(on.pack(gy, transposed=True), gqt)
    for _ in range(3):
        rows.mul_(-1.25)
        layer.add_(0.01)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        q, qt = mx.pack_both(rows)
        y2 = mx.product(q, mx.pack(layer))
        assert torch.equal(gy, y2) and torch.equal(gd, mx.product(mx.pack(y2, transposed=True), qt))


@pytest.mark.parametrize("settings", [{}, {"temperature": 0.0}, {"temperature": 0.7, "top_k": 20, "top_p": 0.9}])
def test_answers(settings):
    """Every step's logits and token against their definitions on the tokens before it."""
    model = example.TiedLanguageModel(500, 64, 256, seed=3)
    answers = example.Answers(model)
    start = torch.tensor([3, 77, 499, 3, 0], device=DEV)
    got = answers.continued(start, 6, seed=5, **settings)
    assert got.shape == (7, 5) and torch.equal(got[0], start)
    assert torch.equal(got, answers.continued(start, 6, seed=5, **settings))
    gen = torch.Generator(device=DEV).manual_seed(5)
    weight, mix = ref.packed_values(model.weight.cpu()), ref.packed_values(model.mix.cpu().t())
    for t in range(6):
        u = torch.rand(5, generator=gen, device=DEV)
        rows = model.weight[got[t]].cpu()
        hidden, bound = ref.product(ref.packed_values(rows), mix, torch.bfloat16)
        own = answers.mx.linear(model.table.lookup(model.weight, got[t]), answers.mix)
        assert language_reference.excess(own, hidden, bound) <= 1.0
        logits = answers.logits(got[t])
        want, bound = ref.product(ref.packed_values(own.cpu()), weight, torch.float32)
        assert language_reference.excess(logits, want, bound) <= 1.0
        for r in range(5):
            tokens, _ = sample_reference.draw(logits[r].double().cpu().numpy(), float(u[r]), **settings)
            assert int(got[t + 1, r]) in tokens


def test_a_trained_model_answers():
    model = example.TiedLanguageModel(300, 64, 512)
    losses = example.train(vocab=300, dim=64, tokens=512, steps=5, model=model)
    assert len(losses) == 5 and all(x == x for x in losses)
    run = example.Answers(model).continued(torch.arange(4, device=DEV), 8, temperature=0.8, top_k=50, top_p=0.95)
    assert run.shape == (9, 4) and int(run.min()) >= 0 and int(run.max()) < 300
