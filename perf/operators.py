"""The language-model operators around the sparsify step, timed and checked:
the lookup of token embeddings and its gradient by sorted tokens, the softmax
cross entropy over the vocabulary and its gradients, and the global norm of a
model's gradients with their clipping into the flat vector that the step reads.

Sizes are those of the package's synthetic workloads (a 50257 x 2048 and a
30522 x 1024 token table, 292 and 391 gradient tensors) and generic ones in
draw().  Token ids follow a log-uniform law (the commonest of 50257 has 6% of
the tokens); hidden states lean towards the target's row by a random amount,
so some targets are nearly certain and others improbable.
"""
import math
import random
import types

import torch

own = False

DEVICE = "cuda"
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
IGNORED = -100
EPS = 1e-6


def _clip(name, layout, n, tensors, dtype, max_norm):
    return {"name": name, "kind": "clip", "layout": layout, "n": n, "tensors": tensors, "dtype": dtype,
            "max_norm": max_norm}


def _table(name, kind, vocab, dim, tokens, dtype, **more):
    return {"name": name, "kind": kind, "vocab": vocab, "dim": dim, "tokens": tokens, "dtype": dtype, **more}


def listed():
    return [
        # a small model's 62 fp32 gradients, 11.7M values, into its flat vector
        _clip("clip_resnet18", "resnet18", 11_689_512, 62, "f32", 1.0),
        # mixed precision: matrices in bf16, the small tensors (norms, biases) in fp32
        _clip("clip_bert_large", "bert_large", 335_141_888, 391, "mixed", 1.0),
        # the largest: every gradient of the GPT model in bf16
        _clip("clip_gpt", "gpt_1p3b", 1_315_723_264, 292, "bf16", 1.0),
        # the tokens of one short prompt: the smallest call, bound by its launch
        _table("lookup_prompt", "lookup", 50257, 2048, 37, "bf16", scale=1.0),
        # a training batch of eight sequences of 2048 positions
        _table("lookup_batch", "lookup", 50257, 2048, 16384, "bf16", scale=45.25),
        # a tied table's second gradient, added to the loss's, fp32, 64 sequences of 512
        _table("lookup_grad_tied", "lookup_grad", 30522, 1024, 32768, "f32", scale=1.0, accumulate=True),
        # the gradient of an untied table, every row written
        _table("lookup_grad_batch", "lookup_grad", 50257, 2048, 16384, "bf16", scale=45.25, accumulate=False),
        # scoring a short continuation: bound by one read of the table
        _table("loss_scoring", "loss", 50257, 2048, 19, "bf16", counted=1.0, mean=False),
        # evaluation of a batch
        _table("loss_batch", "loss", 50257, 2048, 8192, "bf16", counted=1.0, mean=True),
        # a short fine-tuning batch in half precision, prompts not counted, with a loss scale
        _table("loss_grad_short", "loss_grad", 30522, 1024, 300, "f16", counted=0.6, mean=True, scale=1024.0),
        # masked language modelling: 64 sequences of 512, 15% of the positions counted
        _table("loss_grad_masked", "loss_grad", 30522, 1024, 32768, "bf16", counted=0.15, mean=True, scale=1.0),
        # the largest: a training batch of eight sequences of 2048 positions
        _table("loss_grad_batch", "loss_grad", 50257, 2048, 16384, "bf16", counted=1.0, mean=True, scale=1.0),
    ]


def _log_uniform(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    kind = rng.choice(["clip", "clip", "lookup", "lookup_grad", "lookup_grad", "loss", "loss_grad", "loss_grad"])
    if kind == "clip":
        n = _log_uniform(rng, 100_000, 700_000_000)
        return {"kind": kind, "layout": "", "n": n, "tensors": _log_uniform(rng, 1, 400),
                "dtype": rng.choice(["f32", "f16", "bf16", "mixed"]), "max_norm": rng.choice([0.5, 1.0, 1e9])}
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    vocab, dim = _log_uniform(rng, 1000, 70_000), _log_uniform(rng, 64, 4096)
    if rng.random() < 0.6:
        dim = -(-dim // 64) * 64
    tokens = _log_uniform(rng, 1, 20_000)
    # no dearer than the largest listed case
    if kind in ("loss", "loss_grad"):
        most = (1.6e12 if kind == "loss_grad" else 8e11) / (6 if dtype == "f32" else 1)
        tokens = max(1, min(tokens, int(most / (vocab * dim))))
    case = {"kind": kind, "vocab": vocab, "dim": dim, "tokens": tokens, "dtype": dtype}
    if kind in ("loss", "loss_grad"):
        case |= {"counted": rng.choice([1.0, 1.0, 0.15, 0.6]), "mean": rng.random() < 0.7}
    if kind != "loss":
        case["scale"] = {"loss_grad": 256.0 if dtype == "f16" else 1.0}.get(kind, rng.choice([1.0, round(dim ** 0.5, 2)]))
    if kind == "lookup_grad":
        case["accumulate"] = rng.random() < 0.5
    return case


def _resnet18():
    sizes, cin = [64 * 3 * 49, 64, 64], 64
    for planes in (64, 64, 128, 128, 256, 256, 512, 512):
        sizes += [planes * cin * 9, planes, planes, planes * planes * 9, planes, planes]
        if planes != cin:
            sizes += [planes * cin, planes, planes]
        cin = planes
    return sizes + [1000 * 512, 1000]


def _bert_large(h=1024, ffn=4096):
    layer = [h * h, h] * 4 + [h, h, ffn * h, ffn, h * ffn, h, h, h]
    return [30522 * h, 512 * h, 2 * h, h, h] + layer * 24 + [h * h, h]


def _gpt(h=2048, ffn=8192):
    layer = [h, h, 3 * h * h, 3 * h, h * h, h, h, h, h * ffn, ffn, ffn * h, h]
    return [50257 * h, 2048 * h] + layer * 24 + [h, h]


def _sizes(case):
    """(values, counts as a matrix) of every gradient tensor."""
    if case["layout"]:
        sizes = {"resnet18": _resnet18, "bert_large": _bert_large, "gpt_1p3b": _gpt}[case["layout"]]()
        return [(n, n > 8192) for n in sizes]  # norms and biases have at most 8192 values
    n, m = case["n"], case["tensors"]
    r = random.Random(n)
    cuts = sorted(r.sample(range(1, n), m - 1))
    return [(b - a, r.random() < 0.6) for a, b in zip([0] + cuts, cuts + [n])]


def _tensor_type(case, matrix):
    return DTYPE[case["dtype"]] if case["dtype"] != "mixed" else torch.bfloat16 if matrix else torch.float32


def _ids(tokens, vocab, gen):
    u = torch.rand(tokens, generator=gen, device=DEVICE, dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1)).long() - 1).clamp_(0, vocab - 1)


_kept = {}  # the table handle of the last sizes, as a program with one table keeps it


def _handle(case):
    key = tuple(case[k] for k in ("vocab", "dim", "tokens", "dtype"))
    if key not in _kept:
        import paper_2310_00967_amd as micro
        for old in _kept.values():
            torch.cuda.synchronize()
            old.close()
        _kept.clear()
        _kept[key] = micro.TokenTable(case["vocab"], case["dim"], case["tokens"], dtype=DTYPE[case["dtype"]])
    return _kept[key]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    s = types.SimpleNamespace(case=dict(case), kind=case["kind"])
    normal = lambda *shape: torch.empty(shape, device=DEVICE).normal_(generator=gen)  # noqa: E731
    if s.kind == "clip":
        r = random.Random(seed)
        # scales of a model's tensors span three decades; the norm ends well above 1
        s.grads = [normal(n).mul_(math.exp(r.uniform(math.log(1e-5), math.log(1e-2))) * 10).to(_tensor_type(case, m))
                   for n, m in _sizes(case)]
        s.flat = torch.empty(case["n"], device=DEVICE)
        if own:
            import paper_2310_00967_amd as micro
            s.set = micro.GradientSet(s.grads)
        return s
    vocab, dim, tokens, dtype = case["vocab"], case["dim"], case["tokens"], DTYPE[case["dtype"]]
    s.ids = _ids(tokens, vocab, gen)
    if s.kind == "lookup_grad":
        s.grad_out = normal(tokens, dim).mul_(1e-2).to(dtype)
        s.dweight = normal(vocab, dim).mul_(1e-2).to(dtype)
    else:
        s.weight = normal(vocab, dim).mul_(0.02).to(dtype)
    if s.kind in ("loss", "loss_grad"):
        lean = torch.empty(tokens, 1, device=DEVICE).uniform_(0.0, 14.0, generator=gen)
        row = s.weight[s.ids].float()
        s.hidden = (normal(tokens, dim) + lean * row / (row.square().sum(1, keepdim=True) + 1e-6)).to(dtype)
        out = torch.rand(tokens, generator=gen, device=DEVICE) >= case["counted"]
        out[0] = False
        s.targets = s.ids.masked_fill(out, IGNORED)
    if own:
        s.table = _handle(case)
    return s


def _own(s, c):
    if s.kind == "clip":
        norm = s.set.flatten(s.flat, max_norm=c["max_norm"])
        return {"flat": s.flat, "norm": norm}
    if s.kind == "lookup":
        return {"rows": s.table.lookup(s.weight, s.ids, scale=c["scale"])}
    if s.kind == "lookup_grad":
        return {"dweight": s.table.lookup_grad(s.grad_out, s.ids, s.dweight, scale=c["scale"],
                                               accumulate=c["accumulate"])}
    reduction = "mean" if c["mean"] else "sum"
    if s.kind == "loss":
        loss, losses = s.table.loss(s.hidden, s.weight, s.targets, reduction=reduction)
        return {"loss": loss, "losses": losses}
    loss, losses, dhidden, dweight = s.table.loss_grad(s.hidden, s.weight, s.targets, scale=c["scale"],
                                                       reduction=reduction)
    return {"loss": loss, "losses": losses, "dhidden": dhidden, "dweight": dweight}


def run(s):
    c = s.case
    if own:
        return _own(s, c)
    if s.kind == "clip":
        total = sum(g.float().square().sum() for g in s.grads)
        norm = total.sqrt()
        factor = (c["max_norm"] / (norm + EPS)).clamp(max=1.0)
        s.flat.copy_(torch.cat([g.float().reshape(-1) for g in s.grads])).mul_(factor)
        return {"flat": s.flat, "norm": norm}
    if s.kind == "lookup":
        return {"rows": (s.weight[s.ids].float() * c["scale"]).to(s.weight.dtype)}
    if s.kind == "lookup_grad":
        total = torch.zeros(s.dweight.shape, device=DEVICE)
        total.index_add_(0, s.ids, s.grad_out.float())
        total *= c["scale"]
        if c["accumulate"]:
            total += s.dweight.float()
        s.dweight.copy_(total)
        return {"dweight": s.dweight}
    at = (s.targets != IGNORED).nonzero().flatten()
    y, h, w = s.targets[at], s.hidden[at].float(), s.weight.float()
    logits = h @ w.t()
    top = logits.max(1, keepdim=True).values
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    each = (total.log() + top).flatten() - logits.gather(1, y[:, None]).flatten()
    losses = torch.zeros(s.targets.numel(), device=DEVICE)
    losses[at] = each
    loss = each.sum()
    if c["mean"]:
        loss = loss / y.numel()
    if s.kind == "loss":
        return {"loss": loss, "losses": losses}
    p = e / total
    p[torch.arange(y.numel(), device=DEVICE), y] -= 1.0
    p *= c["scale"] / y.numel() if c["mean"] else c["scale"]
    dhidden = torch.zeros_like(s.hidden)
    dhidden[at] = (p @ w).to(dhidden.dtype)
    return {"loss": loss, "losses": losses, "dhidden": dhidden, "dweight": (p.t() @ h).to(s.weight.dtype)}


def _rows(case):
    """The expected number of distinct rows among the tokens of the log-uniform law."""
    v, t = case["vocab"], case["tokens"]
    edges = torch.arange(1, v + 2, dtype=torch.float64).log() / math.log(v + 1)
    return float((1.0 - (1.0 - edges.diff()) ** t).sum())


def work(case):
    """Every input read once and every output written once; the loss's one
    product of tokens and table, three with its gradients, over the counted
    tokens."""
    if case["kind"] == "clip":
        read = sum(n * (4 if _tensor_type(case, m) is torch.float32 else 2) for n, m in _sizes(case))
        return {"bytes": read + 4 * case["n"], "flops": 3 * case["n"]}
    v, d, t, size = case["vocab"], case["dim"], case["tokens"], BYTES[case["dtype"]]
    if case["kind"] == "lookup":
        return {"bytes": 8 * t + (_rows(case) + t) * d * size, "flops": t * d}
    if case["kind"] == "lookup_grad":
        rows = 2 * _rows(case) if case["accumulate"] else v
        return {"bytes": 8 * t + (t + rows) * d * size, "flops": t * d}
    counted = 1 + (t - 1) * case["counted"]
    if case["kind"] == "loss":
        return {"bytes": 12 * t + (counted + v) * d * size, "flops": 2 * counted * v * d}
    return {"bytes": 12 * t + (counted + t + 2 * v) * d * size, "flops": 6 * counted * v * d}


def exact(case, seed):
    """The definitions in 64 bits, token block by token block for the loss."""
    s = prepare(case, seed)
    c = s.case
    if s.kind == "clip":
        square = torch.zeros((), dtype=torch.float64, device=DEVICE)
        for g in s.grads:
            square += torch.linalg.vector_norm(g.double()) ** 2
        norm = math.sqrt(float(square))
        factor = min(1.0, c["max_norm"] / (norm + EPS))
        flat = torch.empty(c["n"], dtype=torch.float64, device=DEVICE)
        at = 0
        for g in s.grads:
            torch.mul(g.double(), factor, out=flat[at:at + g.numel()])
            at += g.numel()
        return {"flat": flat, "norm": norm}
    if s.kind == "lookup":
        return {"rows": torch.nn.functional.embedding(s.ids, s.weight.double()) * c["scale"]}
    if s.kind == "lookup_grad":
        out = s.dweight.double() if c["accumulate"] else torch.zeros_like(s.dweight, dtype=torch.float64)
        order = torch.argsort(s.ids, stable=True)
        names, counts = torch.unique_consecutive(s.ids[order], return_counts=True)
        ends = counts.cumsum(0).tolist()
        first = 0
        for v, end in zip(names.tolist(), ends):
            out[v] += s.grad_out[order[first:end]].double().sum(0) * c["scale"]
            first = end
        return {"dweight": out}
    w, n = s.weight.double(), s.targets.numel()
    counted = int((s.targets >= 0).sum())
    losses = torch.zeros(n, dtype=torch.float64, device=DEVICE)
    dhidden = torch.zeros(s.hidden.shape, dtype=torch.float64, device=DEVICE)
    dweight = torch.zeros_like(w)
    for a in range(0, n, 2048):
        keep = torch.arange(a, min(a + 2048, n), device=DEVICE)
        keep = keep[s.targets[keep] >= 0]
        if not keep.numel():
            continue
        h, y = s.hidden[keep].double(), s.targets[keep]
        logp = torch.log_softmax(torch.mm(h, w.t()), 1)
        losses[keep] = -logp[torch.arange(y.numel(), device=DEVICE), y]
        if s.kind == "loss":
            continue
        d = logp.exp_()
        d.scatter_add_(1, y[:, None], torch.full((y.numel(), 1), -1.0, dtype=torch.float64, device=DEVICE))
        d *= c["scale"] / (counted if c["mean"] else 1)
        dhidden[keep] = torch.mm(d, w)
        dweight += torch.mm(d.t(), h)
    loss = losses.sum() / (counted if c["mean"] else 1)
    if s.kind == "loss":
        return {"loss": loss, "losses": losses}
    return {"loss": loss, "losses": losses, "dhidden": dhidden, "dweight": dweight}
