"""Plain definitions of the language-model operators in 64 bits, on the CPU,
with elementwise bounds of what their kernels' roundings may add.

U[type] is the unit roundoff of a type; EPS that of binary32, in which the
kernels accumulate.
"""
import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# smallest positive number of a type: roundings near zero are absolute
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}
EPS = 2.0 ** -24


def lookup_grad(grad, ids, vocab, scale, old, padding=None):
    """(gradient, bound): m terms of a row are added in binary32 in some fixed
    order (relative error (m + 2) EPS of the sum of magnitudes, scaling and
    adding the old value included), then rounded once."""
    g, ids = grad.double(), ids.long()
    keep = (ids >= 0) & (ids < vocab)
    if padding is not None:
        keep &= ids != padding
    g, ids = g[keep], ids[keep]
    total = torch.zeros(vocab, g.shape[1], dtype=torch.float64).index_add_(0, ids, g)
    mass = torch.zeros_like(total).index_add_(0, ids, g.abs())
    terms = torch.bincount(ids, minlength=vocab).double()[:, None]
    want = scale * total
    if old is not None:
        want = want + old.double()
        mass = mass + old.double().abs() / abs(scale)
    u, tiny = U[grad.dtype], TINY[grad.dtype]
    return want, abs(scale) * (terms + 3) * EPS * mass * (1 + u) + u * want.abs() + tiny


def loss(hidden, weight, targets, mean, ignored=-100):
    """The loss, the tokens' losses and what the gradients need."""
    h, w = hidden.double(), weight.double()
    vocab = w.shape[0]
    y = targets.long()
    keep = (y != ignored) & (y >= 0) & (y < vocab)
    logits = h @ w.t()
    mass = h.abs() @ w.abs().t()
    logp = torch.log_softmax(logits, 1)
    losses = torch.zeros(y.numel(), dtype=torch.float64)
    at = keep.nonzero().flatten()
    losses[at] = -logp[at, y[at]]
    n = int(keep.sum())
    total = losses.sum() / (max(n, 1) if mean else 1)
    # A logit is a binary32 accumulation of D products, each exact (two 16-bit
    # types) or within 6 * 2^-24 (the dropped terms of split binary32); its
    # rounding reaches the loss through the label and through the maximum.  The
    # exponentials and their sum add a few EPS for each unit of a logit's size.
    logit_error = (w.shape[1] + 8) * EPS * mass
    size = logits.abs().max(1).values if vocab else torch.zeros(y.numel(), dtype=torch.float64)
    error = 2 * logit_error.max(1).values + 2.0 ** -20 * (1 + size)
    return {"loss": total, "losses": losses, "error": torch.where(keep, error, torch.zeros_like(error)), "keep": keep,
            "logp": logp, "n": n, "y": y, "mean": mean, "h": h, "w": w, "type": hidden.dtype}


def loss_grads(r, scale, old=None):
    """((dhidden, bound), (dweight, bound)) of what loss() returned.  p - [label]
    carries the logits' error, two roundings to the type (the exponential, then
    its product with the normaliser; binary32 keeps 24 bits) and an underflow
    of binary16 that is below 2^-38; the products add an accumulation of their
    terms, and the output one rounding and that of the factor."""
    u, tiny = U[r["type"]], TINY[r["type"]]
    keep, h, w = r["keep"], r["h"], r["w"]
    factor = scale / (max(r["n"], 1) if r["mean"] else 1)
    p = r["logp"].exp()
    at = keep.nonzero().flatten()
    g = p.clone()
    g[at, r["y"][at]] = torch.expm1(r["logp"][at, r["y"][at]])
    off = p * r["error"][:, None] + 2.1 * u * p + 2.0 ** -38
    # at the label the two roundings are of p - 1 itself
    off[at, r["y"][at]] = (p[at, r["y"][at]] * r["error"][at] + (2.1 * u + 2.0 ** -20) * g[at, r["y"][at]].abs()
                           + 2.0 ** -20 * r["error"][at] + 2.0 ** -38)
    g, off = g * keep[:, None], off * keep[:, None]
    dh, dw = factor * (g @ w), factor * (g.t() @ h)
    mass_h, mass_w = g.abs() @ w.abs(), g.abs().t() @ h.abs()
    bound_h = abs(factor) * (off @ w.abs() + (w.shape[0] + 16) * EPS * mass_h)
    bound_w = abs(factor) * (off.t() @ h.abs() + (h.shape[0] + 16) * EPS * mass_w)
    if old is not None:
        dw = dw + old.double()
    return ((dh, bound_h * (1 + u) + (u + 4 * EPS) * dh.abs() + tiny),
            (dw, bound_w * (1 + u) + (u + 4 * EPS) * dw.abs() + tiny))


def excess(got, want, bound):
    """The largest |got - want| / bound; NaN and infinities have to be equal."""
    got = got.detach().cpu().double()
    assert got.shape == want.shape
    fine = want.isfinite()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got[~fine & ~want.isnan()], want[~fine & ~want.isnan()])
    if not bool(fine.any()):
        return 0.0
    return float(((got - want).abs() / bound.clamp(min=1e-300))[fine].max())
