"""The softmax cross entropy over a token table and its gradients on the GPU,
against the definition in 64 bits within derived elementwise bounds."""
import math

import pytest
import torch

import paper_2310_00967_amd as micro
from paper_2310_00967_amd import _lib

import language_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]


def make(vocab, dim, tokens, dtype, seed=0, counted=1.0, lean=8.0):
    """Hidden rows that lean towards their target's row by 0 to `lean` units of
    logit, targets of which a share counts."""
    gen = torch.Generator().manual_seed(seed + 31 * vocab + tokens)
    weight = torch.randn(vocab, dim, generator=gen).mul_(dim ** -0.5).to(dtype)
    y = torch.randint(0, vocab, (tokens,), generator=gen)
    row = weight[y].float()
    push = torch.rand(tokens, 1, generator=gen) * lean
    hidden = (torch.randn(tokens, dim, generator=gen) + push * row / (row.square().sum(1, keepdim=True) + 1e-3)).to(dtype)
    out = torch.rand(tokens, generator=gen) >= counted
    return hidden, weight, y.masked_fill(out, -100)


def check(table, hidden, weight, targets, reduction="mean", scale=1.0, old=None, ignored=-100):
    """Both calls against the definition; returns the loss call's tensors."""
    h, w, y = hidden.to(DEV), weight.to(DEV), targets.to(DEV)
    r = ref.loss(hidden, weight, targets, reduction == "mean", ignored)
    loss, losses = table.loss(h, w, y, reduction=reduction)
    assert loss.dtype == F32 and losses.dtype == F32 and losses.shape == targets.shape
    total = r["error"].sum() / (max(r["n"], 1) if r["mean"] else 1) + 2 * ref.EPS * r["loss"].abs()
    slack = r["error"] + 2 * ref.EPS * r["losses"].abs() + 1e-300
    assert ref.excess(losses, r["losses"], slack) <= 1.0
    assert ref.excess(loss, r["loss"], total + 1e-300) <= 1.0
    dweight = None if old is None else old.to(DEV)
    got = table.loss_grad(h, w, y, scale=scale, reduction=reduction, dweight=dweight, accumulate=old is not None)
    assert ref.excess(got[1], r["losses"], slack) <= 1.0
    assert ref.excess(got[0], r["loss"], total + 1e-300) <= 1.0
    (dh, dh_bound), (dw, dw_bound) = ref.loss_grads(r, scale, old)
    assert got[2].shape == hidden.shape and got[2].dtype == hidden.dtype
    assert ref.excess(got[2], dh, dh_bound) <= 1.0, "dhidden"
    assert ref.excess(got[3], dw, dw_bound) <= 1.0, "dweight"
    return got


SIZES = [(1, 1, 1), (2, 3, 1), (5, 8, 3), (33, 64, 31), (63, 64, 32), (64, 128, 33), (65, 77, 64), (130, 40, 65),
         (1000, 64, 7), (300, 200, 257), (5003, 128, 40), (777, 576, 600), (257, 1, 300), (2000, 100, 1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,dim,tokens", SIZES)
def test_sizes(dtype, vocab, dim, tokens):
    table = micro.TokenTable(vocab, dim, tokens, dtype=dtype)
    check(table, *make(vocab, dim, tokens, dtype), scale=64.0)
    table.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [20, 50, 400])
@pytest.mark.parametrize("counted", [0.0, 0.02, 0.5])
def test_tokens_that_do_not_count(dtype, tokens, counted):
    table = micro.TokenTable(150, 72, tokens, dtype=dtype)
    hidden, weight, targets = make(150, 72, tokens, dtype, counted=counted)
    got = check(table, hidden, weight, targets, scale=8.0)
    idle = targets == -100
    assert bool((got[2].cpu()[idle] == 0).all()) and bool((got[1].cpu()[idle] == 0).all())
    if counted == 0.0:
        assert float(got[0]) == 0.0 and bool((got[3] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("reduction", ["sum", "mean"])
def test_reduction_and_accumulation(dtype, reduction):
    table = micro.TokenTable(200, 96, 130, dtype=dtype)
    hidden, weight, targets = make(200, 96, 130, dtype, counted=0.8)
    old = torch.randn(200, 96, generator=torch.Generator().manual_seed(9)).to(dtype)
    check(table, hidden, weight, targets, reduction=reduction, scale=0.5, old=old)
    check(table, hidden, weight, torch.full_like(targets, -100), reduction=reduction, scale=0.5, old=old)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counted", [0.1, 0.5, 1.0])
def test_several_token_blocks(dtype, counted):
    """Scratch for 256 tokens' scores, 1000 tokens: four blocks, of which some
    have nothing counted."""
    table = micro.TokenTable(300, 136, 1000, dtype=dtype, score_bytes=1)
    check(table, *make(300, 136, 1000, dtype, counted=counted), scale=16.0)
    hidden, weight, targets = make(300, 136, 1000, dtype, seed=4, counted=counted)
    old = torch.randn(300, 136, generator=torch.Generator().manual_seed(9)).to(dtype)
    check(table, hidden, weight, targets, old=old)
    check(table, hidden[:90], weight, targets[:90], old=old)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [257, 300, 384, 385])
def test_short_calls_of_several_token_blocks(dtype, tokens):
    """Blocks of 256 tokens at lengths on both sides of where the tiles change."""
    table = micro.TokenTable(200, 72, tokens, dtype=dtype, score_bytes=1)
    check(table, *make(200, 72, tokens, dtype, counted=0.95), scale=8.0)


def chunked(hidden, weight, targets, rows):
    """Losses of all tokens in 64 bits on the GPU, dhidden of the last tokens and
    dweight of the given rows, in chunks of tokens (sum reduction)."""
    h, w = hidden.double(), weight.double()
    losses, dw = [], torch.zeros(len(rows), w.shape[1], dtype=torch.float64, device=DEV)
    for a in range(0, h.shape[0], 4096):
        y = targets[a:a + 4096]
        logp = torch.log_softmax(h[a:a + 4096] @ w.t().contiguous(), 1)
        losses.append(-logp.gather(1, y[:, None]).flatten())
        g = logp[:, rows].exp() - (y[:, None] == rows[None, :]).double()
        dw += g.t().contiguous() @ h[a:a + 4096]
    g = logp.exp()
    g[torch.arange(y.numel(), device=DEV), y] -= 1.0
    return torch.cat(losses), g @ w, dw


@pytest.mark.parametrize("vocab,dim,tokens,score_bytes", [(65_537, 64, 66_000, 9 << 30),  # 4.3e9 scores in one block
                                                          (40, 8, 1_200_000, 2 << 30)])  # more rows than a grid's y
def test_offsets_and_grids_past_their_limits(vocab, dim, tokens, score_bytes):
    """Against 64 bits to 2% of the largest gradient (each value carries three
    roundings of 2^-8; a wrong offset is off by all of it), losses to 1e-4."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    weight = torch.randn(vocab, dim, generator=gen, device=DEV).mul_(dim ** -0.5).bfloat16()
    hidden = torch.randn(tokens, dim, generator=gen, device=DEV).bfloat16()
    targets = torch.randint(0, vocab, (tokens,), generator=gen, device=DEV)
    table = micro.TokenTable(vocab, dim, tokens, dtype=BF16, score_bytes=score_bytes)
    loss, losses, dh, dw = table.loss_grad(hidden, weight, targets, reduction="sum")
    rows = torch.tensor([0, 1, vocab // 2, vocab - 2, vocab - 1], device=DEV)
    want, want_h, want_w = chunked(hidden, weight, targets, rows)
    assert float((losses.double() - want).abs().max()) <= 1e-4
    assert abs(float(loss) / float(want.sum()) - 1) <= 1e-6
    last = want_h.shape[0]
    assert float((dh[-last:].double() - want_h).abs().max()) <= 0.02 * float(want_h.abs().max())
    assert float((dw[rows].double() - want_w).abs().max()) <= 0.02 * float(want_w.abs().max())
    table.close()


@pytest.mark.parametrize("dtype", TYPES)
def test_calls_of_different_lengths_on_one_handle(dtype):
    table = micro.TokenTable(400, 64, 900, dtype=dtype, score_bytes=400 * 2 * 512)
    for tokens in (900, 1, 33, 513, 64, 0, 256, 300, 20):
        check(table, *make(400, 64, tokens, dtype, seed=tokens, counted=0.9), scale=4.0)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("tokens", [16, 60, 1100])
def test_a_product_of_few_tiles_is_split_along_the_sum(dtype, tokens):
    """One tile of output and a long sum (over the vocabulary, over tokens)."""
    check(micro.TokenTable(9001, 64, tokens, dtype=dtype), *make(9001, 64, tokens, dtype), scale=32.0)
    check(micro.TokenTable(40, 64, 4 * tokens, dtype=dtype), *make(40, 64, 4 * tokens, dtype), scale=32.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,dim,tokens,counted", [(129, 1024, 1, 1.0), (1549, 2304, 7, 1.0), (700, 1100, 32, 0.1),
                                                      (1000, 1500, 33, 1.0), (640, 2000, 200, 0.3), (300, 4096, 384, 1.0),
                                                      (900, 1024, 90, 0.0)])
def test_scores_of_few_tiles_are_split_along_the_width(dtype, vocab, dim, tokens, counted):
    table = micro.TokenTable(vocab, dim, tokens, dtype=dtype)
    check(table, *make(vocab, dim, tokens, dtype, counted=counted), scale=32.0)
    table.close()


@pytest.mark.parametrize("dtype", TYPES)
def test_strided_rows_and_shapes(dtype):
    hidden, weight, targets = make(90, 64, 60, dtype)
    table = micro.TokenTable(90, 64, 60, dtype=dtype)
    wide_h = torch.zeros(60, 80, dtype=dtype, device=DEV)
    wide_w = torch.zeros(90, 75, dtype=dtype, device=DEV)
    wide_h[:, 7:71] = hidden.to(DEV)
    wide_w[:, 3:67] = weight.to(DEV)
    dh = torch.full((60, 70), 3.0, dtype=dtype, device=DEV)
    dw = torch.full((90, 66), 3.0, dtype=dtype, device=DEV)
    loss, losses, _, _ = table.loss_grad(wide_h[:, 7:71], wide_w[:, 3:67], targets.int().to(DEV), dhidden=dh[:, 1:65],
                                         dweight=dw[:, 2:66])
    r = ref.loss(hidden, weight, targets, True)
    (want_h, bound_h), (want_w, bound_w) = ref.loss_grads(r, 1.0)
    assert ref.excess(dh[:, 1:65], want_h, bound_h) <= 1.0 and ref.excess(dw[:, 2:66], want_w, bound_w) <= 1.0
    for t, a, b in ((dh, 1, 65), (dw, 2, 66)):
        assert bool((t[:, :a] == 3.0).all()) and bool((t[:, b:] == 3.0).all())
    # hidden states of a batch of sequences
    shaped = table.loss_grad(hidden.view(5, 12, 64).to(DEV), weight.to(DEV), targets.view(5, 12).to(DEV))
    assert shaped[1].shape == (5, 12) and shaped[2].shape == (5, 12, 64)
    assert torch.equal(shaped[1].flatten(), losses) and torch.equal(shaped[2].view(60, 64), dh[:, 1:65])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [30.0, 3000.0])
def test_large_logits(dtype, size):
    """Nearly certain and hopeless tokens: exponentials that underflow, p - 1
    that cancels."""
    hidden, weight, targets = make(500, 64, 90, dtype, lean=0.0)
    hidden = (hidden.float() * size / 8).to(dtype)
    table = micro.TokenTable(500, 64, 90, dtype=dtype)
    h, w, y = hidden.to(DEV), weight.to(DEV), targets.to(DEV)
    r = ref.loss(hidden, weight, targets, True)
    loss, losses, dh, dw = table.loss_grad(h, w, y)
    slack = r["error"] + 2 * ref.EPS * r["losses"].abs()
    assert ref.excess(losses, r["losses"], slack) <= 1.0
    if size < 100:
        (want_h, bound_h), (want_w, bound_w) = ref.loss_grads(r, 1.0)
        assert ref.excess(dh, want_h, bound_h) <= 1.0 and ref.excess(dw, want_w, bound_w) <= 1.0
    assert bool(dh.isfinite().all()) and bool(dw.isfinite().all())


def test_a_nearly_certain_token_keeps_its_gradient():
    """p = 1 - 1e-4: in bfloat16 p itself would round to 1."""
    weight = torch.zeros(8, 64, dtype=BF16)
    weight[0, 0], weight[1, 0] = 1.0, -1.0
    hidden = torch.zeros(40, 64, dtype=BF16)
    hidden[:, 0] = 8.0
    targets = torch.zeros(40, dtype=torch.int64)
    table = micro.TokenTable(8, 64, 40, dtype=BF16)
    loss, _, dh, dw = table.loss_grad(hidden.to(DEV), weight.to(DEV), targets.to(DEV), reduction="sum")
    r = ref.loss(hidden, weight, targets, False)
    (want_h, _), (want_w, _) = ref.loss_grads(r, 1.0)
    assert float(want_w[0, 0]) < -1e-4
    assert abs(float(dw[0, 0]) / float(want_w[0, 0]) - 1) < 0.02
    assert abs(float(dh[0, 0]) / float(want_h[0, 0]) - 1) < 0.02


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_values_that_are_not_finite(dtype, bad):
    """A token whose hidden state is not finite has a NaN loss and gradient;
    the other tokens' own results are as without it."""
    hidden, weight, targets = make(200, 64, 80, dtype)
    table = micro.TokenTable(200, 64, 80, dtype=dtype)
    clean = table.loss_grad(hidden.to(DEV), weight.to(DEV), targets.to(DEV), reduction="sum")
    hidden[17, 5] = bad
    loss, losses, dh, dw = table.loss_grad(hidden.to(DEV), weight.to(DEV), targets.to(DEV), reduction="sum")
    assert bool(losses[17].isnan()) and bool(loss.isnan()) and bool(dh[17].isnan().all())
    keep = torch.arange(80, device=DEV) != 17
    assert torch.equal(losses[keep], clean[1][keep]) and torch.equal(dh[keep], clean[2][keep])
    targets[17] = -100  # and where it does not count it has no part at all
    loss, losses, dh, dw = table.loss_grad(hidden.to(DEV), weight.to(DEV), targets.to(DEV), reduction="sum")
    assert bool(loss.isfinite()) and float(losses[17]) == 0.0 and bool((dh[17] == 0).all()) and bool(dw.isfinite().all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("low", ["lowest", -math.inf])
def test_a_masked_vocabulary(dtype, low):
    """Rows that push their logits to the type's lowest values, or to -inf,
    have no part."""
    hidden, weight, targets = make(300, 64, 70, dtype)
    hidden[:, 0] = 1.0
    weight[:, 0] = 0.0
    low = torch.finfo(dtype).min if low == "lowest" else low
    weight[100:250] = 0.0
    weight[100:250, 0] = low
    targets = targets % 100
    table = micro.TokenTable(300, 64, 70, dtype=dtype)
    loss, losses, dh, dw = table.loss_grad(hidden.to(DEV), weight.to(DEV), targets.to(DEV), reduction="sum")
    rest = torch.cat([weight[:100], weight[250:]])
    r = ref.loss(hidden, rest, targets, False)
    assert ref.excess(losses, r["losses"], r["error"] + 2 * ref.EPS * r["losses"].abs()) <= 1.0
    assert bool((dw[100:250] == 0).all())


def test_targets_outside_the_vocabulary():
    hidden, weight, targets = make(50, 64, 40, F32)
    targets[3], targets[9] = 50, -7
    table = micro.TokenTable(50, 64, 40)
    loss, losses, dh, dw = table.loss_grad(hidden.to(DEV), weight.to(DEV), targets.to(DEV), reduction="sum")
    out = torch.tensor([3, 9])
    assert bool(loss.isnan()) and bool(losses.cpu()[out].isnan().all()) and bool((dh.cpu()[out] == 0).all())
    r = ref.loss(hidden, weight, targets, False)
    (want_h, bound_h), (want_w, bound_w) = ref.loss_grads(r, 1.0)
    assert ref.excess(dh, want_h, bound_h) <= 1.0 and ref.excess(dw, want_w, bound_w) <= 1.0
    assert int(losses.isnan().sum()) == 2
    other = micro.TokenTable(50, 64, 40, ignore_id=-7)
    check(other, hidden, weight, targets.masked_fill(targets == 50, -7), ignored=-7)


@pytest.mark.parametrize("dtype", TYPES)
def test_results_do_not_change_between_runs(dtype):
    hidden, weight, targets = make(3000, 128, 500, dtype)
    table = micro.TokenTable(3000, 128, 500, dtype=dtype)
    args = (hidden.to(DEV), weight.to(DEV), targets.to(DEV))
    first = table.loss_grad(*args)
    for _ in range(4):
        for a, b in zip(first, table.loss_grad(*args)):
            assert torch.equal(a, b)


def test_gradients_are_the_derivatives():
    """Central differences of the definition's loss in 64 bits along random
    directions: the step of 1e-4 leaves 1e-7 of curvature, the binary32
    gradients 1e-5."""
    hidden, weight, targets = make(120, 32, 24, F32, counted=0.8)
    table = micro.TokenTable(120, 32, 24)
    _, _, dh, dw = table.loss_grad(hidden.to(DEV), weight.to(DEV), targets.to(DEV), scale=3.0)
    gen = torch.Generator().manual_seed(1)
    value = lambda h, w: 3.0 * float(ref.loss(h, w, targets, True)["loss"])  # noqa: E731
    for _ in range(4):
        a = torch.randn(hidden.shape, generator=gen, dtype=torch.float64)
        b = torch.randn(weight.shape, generator=gen, dtype=torch.float64)
        h, w, e = hidden.double(), weight.double(), 1e-4
        slope = (value(h + e * a, w) - value(h - e * a, w)) / (2 * e)
        got = float((dh.cpu().double() * a).sum())
        assert abs(slope - got) <= 1e-5 * float((dh.cpu().double().abs() * a.abs()).sum()) + 1e-7
        slope = (value(h, w + e * b) - value(h, w - e * b)) / (2 * e)
        got = float((dw.cpu().double() * b).sum())
        assert abs(slope - got) <= 1e-5 * float((dw.cpu().double().abs() * b.abs()).sum()) + 1e-7


def test_another_stream_and_a_graph():
    stream = torch.cuda.Stream()
    hidden, weight, targets = make(300, 64, 100, BF16)
    table = micro.TokenTable(300, 64, 100, dtype=BF16, stream=stream)
    h, w, y = hidden.to(DEV), weight.to(DEV), targets.to(DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        table.loss_grad(h, w, y)  # the scratch
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = table.loss_grad(h, w, y)
    for seed in range(3):
        hidden, weight, targets = make(300, 64, 100, BF16, seed=seed, counted=0.5 + 0.2 * seed)
        h.copy_(hidden), w.copy_(weight), y.copy_(targets)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = table.loss_grad(h, w, y)
        stream.synchronize()
        for a, b in zip(got, eager):
            assert torch.equal(a, b)


def test_refusals():
    hidden, weight, targets = (t.to(DEV) for t in make(60, 64, 20, F32))
    table = micro.TokenTable(60, 64, 20)
    dh = torch.full((20, 64), 7.0, device=DEV)
    dw = torch.full((60, 64), 7.0, device=DEV)
    more = torch.zeros(21, dtype=torch.int64, device=DEV)
    bad = [lambda: table.loss(hidden, weight, targets.float()), lambda: table.loss(hidden[:19], weight, targets),
           lambda: table.loss(hidden.half(), weight, targets), lambda: table.loss(hidden, weight[:59], targets),
           lambda: table.loss(hidden, weight, targets, reduction="none"),
           lambda: table.loss(torch.zeros(21, 64, device=DEV), weight, more),
           lambda: table.loss_grad(hidden, weight, targets, scale=math.inf, dhidden=dh, dweight=dw),
           lambda: table.loss_grad(hidden, weight, targets, scale=1e300, dhidden=dh, dweight=dw),
           lambda: table.loss_grad(hidden, weight, targets, accumulate=True),
           lambda: table.loss_grad(hidden, weight, targets, dhidden=hidden, dweight=dw),
           lambda: table.loss_grad(hidden, weight, targets, dhidden=dh, dweight=weight),
           lambda: table.loss_grad(hidden, weight, targets, dhidden=dh[:, :32], dweight=dw)]
    for call in bad:
        with pytest.raises((TypeError, ValueError, _lib.MicroError)):
            call()
    torch.cuda.synchronize()
    assert bool((dh == 7).all()) and bool((dw == 7).all())
    huge = micro.TokenTable(2 ** 22 + 1, 1, 4)
    with pytest.raises(_lib.MicroError) as e:
        huge.loss(torch.zeros(4, 1, device=DEV), torch.zeros(2 ** 22 + 1, 1, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV))
    assert e.value.status == _lib.MICRO_ERANGE
    table.close()
    with pytest.raises(RuntimeError):
        table.loss(hidden, weight, targets)
