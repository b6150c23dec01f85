"""How often the token loss rounds to 16 bits on the way to its gradients.

The gradients' operands are 16-bit, so p - [label] is rounded once, and the
output once.  The kernels' error against 64 bits is compared, in root mean
square over all values, with that of two computations in 64 bits: one that
rounds p once, and one that rounds the exponentials before it too."""
import pytest
import torch

import paper_2310_00967_amd as micro

pytestmark = pytest.mark.gpu

DEV = "cuda"


def rms(x):
    return float(x.square().mean().sqrt())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("vocab,dim,tokens,score_bytes", [(600, 128, 200, None), (1200, 192, 700, None), (900, 128, 600, 1)])
def test_logit_gradients_are_rounded_once(dtype, vocab, dim, tokens, score_bytes):
    """Every target is row 0, whose values are zero, so no rounding at a label
    reaches dhidden; dweight is compared in the other rows.  Exponents held in
    16 bits with a step of at most 1/1800 within 2^8 of a group's maximum add
    less than an eighth of what a rounding of the exponentials adds in square;
    the bound is half of what that rounding adds."""
    gen = torch.Generator().manual_seed(vocab)
    weight = torch.randn(vocab, dim, generator=gen).mul_(1.5 * dim ** -0.5)
    weight[0] = 0.0
    weight = weight.to(dtype)
    hidden = torch.randn(tokens, dim, generator=gen).to(dtype)
    targets = torch.zeros(tokens, dtype=torch.int64)
    table = micro.TokenTable(vocab, dim, tokens, dtype=dtype, score_bytes=score_bytes)
    _, _, dh, dw = table.loss_grad(hidden.to(DEV), weight.to(DEV), targets.to(DEV), reduction="sum")
    h, w = hidden.double(), weight.double()
    logits = h @ w.t()
    p = torch.softmax(logits, 1)
    unit = 2.0 ** 14 if dtype is torch.float16 else 1.0  # binary16 holds these values times this
    held = lambda x: (x * unit).to(dtype).double() / unit  # noqa: E731
    # exponentials against the greatest of each 64 rows
    top = torch.cat([g.max(1, keepdim=True).values.expand_as(g) for g in logits.split(64, 1)], 1)
    twice = held(held((logits - top).exp()) * (top - logits.logsumexp(1, keepdim=True)).exp())
    for got, product in ((dh, lambda g: g @ w), (dw[1:], lambda g: g.t()[1:] @ h)):
        exact = product(p)  # (row 0 has no part in either)
        error = [rms(product(g).to(dtype).double() - exact) for g in (held(p), twice)]
        assert error[1] > 1.02 * error[0]
        assert rms(got.cpu().double() - exact) <= error[0] + 0.5 * (error[1] - error[0])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("vocab,dim,tokens,score_bytes", [(600, 128, 200, None), (1200, 200, 700, None), (900, 72, 600, 1),
                                                          (9001, 64, 60, None)])
@pytest.mark.parametrize("counted", [1.0, 0.6])
def test_the_labels_rounding_does_not_reach_dhidden(dtype, vocab, dim, tokens, score_bytes, counted):
    """The label's p - 1 is most of a token's gradient.  dhidden is as near to 64
    bits as where only p is rounded, and not where p - 1 is too: the bound is
    half of what the latter adds."""
    gen = torch.Generator().manual_seed(vocab)
    weight = torch.randn(vocab, dim, generator=gen).mul_(dim ** -0.5).to(dtype)
    targets = torch.randint(0, vocab, (tokens,), generator=gen)
    row = weight[targets].float()
    lean = torch.rand(tokens, 1, generator=gen) * 12.0  # the label's p from nearly 0 to nearly 1
    hidden = (torch.randn(tokens, dim, generator=gen) + lean * row / row.square().sum(1, keepdim=True)).to(dtype)
    targets[torch.rand(tokens, generator=gen) >= counted] = -100
    table = micro.TokenTable(vocab, dim, tokens, dtype=dtype, score_bytes=score_bytes)
    dh = table.loss_grad(hidden.to(DEV), weight.to(DEV), targets.to(DEV), reduction="sum")[2]
    keep = (targets >= 0).nonzero().flatten()
    h, w, y = hidden[keep].double(), weight.double(), targets[keep]
    unit = 2.0 ** 14 if dtype is torch.float16 else 1.0
    held = lambda x: (x * unit).to(dtype).double() / unit  # noqa: E731
    logp = torch.log_softmax(h @ w.t(), 1)
    g = logp.exp()
    at = torch.arange(y.numel())
    g[at, y] = torch.expm1(logp[at, y])
    exact = g @ w
    both = held(g)
    only_p = both.clone()
    only_p[at, y] = g[at, y]
    error = [rms((x @ w).to(dtype).double() - exact) for x in (only_p, both)]
    assert error[1] > 1.02 * error[0]
    assert rms(dh.cpu()[keep].double() - exact) <= error[0] + 0.5 * (error[1] - error[0])
