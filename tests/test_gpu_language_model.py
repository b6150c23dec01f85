"""The operators together, as examples/tied_language_model.py runs them: its
gradients against automatic differentiation in 64 bits, and its training."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("tied_language_model",
                                                  os.path.join(ROOT, "examples", "tied_language_model.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradients_of_the_whole_model():
    """Each bfloat16 rounding on the way (rows, hidden, both gradients of the
    hidden rows, the logit gradients, the table's gradient twice) is 2^-8 of
    its value at most: eight of them, against the largest gradient."""
    module = example()
    model = module.TiedLanguageModel(300, 64, 500, seed=3)
    x, y = next(module.batches(300, 500, 4))
    loss = model.gradients(x, y)
    w = model.weight.double().cpu().requires_grad_()
    m = model.mix.double().cpu().requires_grad_()
    want = torch.nn.functional.cross_entropy(w[x.cpu()] @ m @ w.t(), y.cpu())
    want.backward()
    want = float(want.detach())
    assert abs(float(loss) - want) <= 8 * 2.0 ** -8 * want
    for got, exact in ((model.dweight, w.grad), (model.dmix, m.grad)):
        off = (got.double().cpu() - exact).abs().max()
        assert float(off) <= 8 * 2.0 ** -8 * float(exact.abs().max())
    flat = torch.empty(model.params.numel(), device="cuda")
    norm = float(model.grads.flatten(flat, max_norm=1e-3))
    assert abs(float(flat.double().norm()) - 1e-3) <= 1e-3 * 2e-3  # the 1e-6 in the factor's denominator included
    both = torch.cat([model.dweight.flatten().double(), model.dmix.flatten().double()])
    assert abs(norm / float(both.norm()) - 1) <= 1e-6


def test_training_learns_the_chain():
    losses = example().train(vocab=500, dim=64, tokens=2048, steps=150)
    assert losses[0] > 5.0
    assert sum(losses[-10:]) / 10 < 0.6 * losses[0]
