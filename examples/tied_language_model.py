"""A small tied-embedding language model trained by one worker with MiCRO's
sparsified gradients, from token ids to the sparse model update:

    rows    = table.lookup(weight, x)                   token rows
    hidden  = rows @ mix                                (the rest of the model)
    loss    = table.loss_grad(hidden, weight, y)        loss and both gradients
    dweight += table.lookup_grad(drows, x)              the table's other gradient
    grads.flatten(flat, max_norm)                       global norm, clipped, one vector
    sp.ef_step(flat * rate, residual, ...)              the worker's sparsified step
    sp.sparse_update(params, idx, val, world)           the model update

    table.sample(mx.linear(hidden, packed table))       and its answers, from weights in 4 bits

The weights of the forward pass are bfloat16 copies of one flat binary32
vector, which the updates go to.  The data is a synthetic chain: a token's
successor is a fixed random one nine times out of ten, else any.

    python examples/tied_language_model.py [--steps 200] [--vocab 2000] [--dim 128] [--answer 16]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2310_00967_amd as micro  # noqa: E402


class TiedLanguageModel:
    """The token table and a square mixing matrix, as one flat vector."""

    def __init__(self, vocab, dim, tokens, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.vocab, self.dim = vocab, dim
        shapes = [(vocab, dim), (dim, dim)]
        sizes = [math.prod(s) for s in shapes]
        self.params = torch.empty(sum(sizes), device=device)
        views = [v.view(s) for v, s in zip(self.params.split(sizes), shapes)]
        views[0].normal_(0.0, dim ** -0.5, generator=gen)
        views[1].normal_(0.0, dim ** -0.5, generator=gen)
        self.views = views
        self.weight, self.mix = (v.bfloat16() for v in views)
        # gradients that the operators write and the set reads, step after step
        self.dweight, self.dmix = torch.empty_like(self.weight), torch.empty_like(views[1])
        self.table = micro.TokenTable(vocab, dim, tokens, dtype=torch.bfloat16)
        self.grads = micro.GradientSet([self.dweight, self.dmix])

    def gradients(self, x, y):
        """Loss of predicting y from x; fills the gradient tensors."""
        rows = self.table.lookup(self.weight, x)
        hidden = rows @ self.mix
        loss, _, dhidden, _ = self.table.loss_grad(hidden, self.weight, y, dweight=self.dweight)
        torch.matmul(rows.float().t(), dhidden.float(), out=self.dmix)
        drows = dhidden @ self.mix.t().contiguous()
        self.table.lookup_grad(drows, x, self.dweight, accumulate=True)
        return loss

    def refresh(self):
        """The forward pass's copies after an update of params."""
        self.weight.copy_(self.views[0])
        self.mix.copy_(self.views[1])


def batches(vocab, tokens, seed, device="cuda"):
    gen = torch.Generator(device=device).manual_seed(seed)
    successor = torch.randperm(vocab, generator=gen, device=device)
    while True:
        x = torch.randint(0, vocab, (tokens,), generator=gen, device=device)
        any_token = torch.randint(0, vocab, (tokens,), generator=gen, device=device)
        keep = torch.rand(tokens, generator=gen, device=device) < 0.9
        yield x, torch.where(keep, successor[x], any_token)


class Answers:
    """Continuations of a trained model, whose weights are packed to 4 bits."""

    def __init__(self, model):
        self.model, self.mx = model, micro.Microscaled()
        self.weight = self.mx.pack(model.weight)
        self.mix = self.mx.pack(model.mix, transposed=True)  # rows @ mix is rows (mix^T)^T

    def logits(self, tokens):
        rows = self.model.table.lookup(self.model.weight, tokens)
        hidden = self.mx.linear(rows, self.mix)
        return self.mx.linear(hidden, self.weight, dtype=torch.float32)

    def continued(self, tokens, length, seed=0, **settings):
        """Tokens (one a continuation) followed by `length` drawn ones: int64, (length +
        1, continuations).  settings: those of TokenTable.sample."""
        gen = torch.Generator(device=tokens.device).manual_seed(seed)
        out = [tokens]
        for _ in range(length):
            u = torch.rand(tokens.numel(), generator=gen, device=tokens.device)
            ids, _ = self.model.table.sample(self.logits(out[-1]), u, **settings)
            out.append(ids)
        return torch.stack(out)


def train(vocab=2000, dim=128, tokens=4096, steps=200, rate=100.0, max_norm=0.05, density=0.05, seed=0, report=None, model=None):
    """Trains (a model of the given sizes, or a new one) and returns the losses of every
    step."""
    model = model if model is not None else TiedLanguageModel(vocab, dim, tokens, seed)
    n = model.params.numel()
    sp = micro.Sparsifier(n)
    flat, residual = torch.empty(n, device="cuda"), torch.zeros(n, device="cuda")
    theta, losses = None, []
    data = batches(vocab, tokens, seed + 1)
    for t in range(steps):
        x, y = next(data)
        loss = model.gradients(x, y)
        norm = model.grads.flatten(flat, max_norm=max_norm)
        flat.mul_(rate)
        if theta is None:  # a start at the target density
            theta = float(flat.abs().kthvalue(n - int(density * n)).values)
        k, theta, _, idx, val = sp.ef_step(flat, residual, t, 0, 1, density, theta)
        sp.sparse_update(model.params, idx, val, 1)
        model.refresh()
        losses.append(float(loss))
        if report and (t % report == 0 or t == steps - 1):
            print(f"step {t}: loss {losses[-1]:.4f}, gradient norm {float(norm):.4f}, {k / n:.3%} of {n} values sent",
                  flush=True)
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--vocab", type=int, default=2000)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--answer", type=int, default=16, help="tokens to continue with after the training")
    a = ap.parse_args()
    trained = TiedLanguageModel(a.vocab, a.dim, a.tokens)
    train(vocab=a.vocab, dim=a.dim, tokens=a.tokens, steps=a.steps, report=max(1, a.steps // 10), model=trained)
    if a.answer > 0:
        starts = torch.arange(4, device="cuda")
        for run in Answers(trained).continued(starts, a.answer, temperature=0.8, top_k=50, top_p=0.95).t().tolist():
            print(" ".join(map(str, run)))
