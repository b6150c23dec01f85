"""The token table's lookup and its gradient on the GPU, against their
definitions: the lookup bit for bit, the gradient within its derived bound."""
import pytest
import torch

import paper_2310_00967_amd as micro
from paper_2310_00967_amd import _lib

import language_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def draw_ids(tokens, vocab, kind, gen):
    if kind == "one":
        return torch.full((tokens,), vocab // 2)
    if kind == "skewed":
        u = torch.rand(tokens, generator=gen, dtype=torch.float64)
        return (torch.exp(u * torch.tensor(float(vocab + 1)).log()).long() - 1).clamp(0, vocab - 1)
    return torch.randint(0, vocab, (tokens,), generator=gen)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,dim,tokens,scale", [(1, 1, 1, 1.0), (7, 3, 5, 2.5), (100, 64, 33, 1.0), (513, 77, 300, 8.7),
                                                    (1000, 1024, 65, 32.0), (50, 4099, 9, 0.1), (3000, 8, 20000, 1.0)])
@pytest.mark.parametrize("ids_type", [torch.int64, torch.int32])
def test_lookup(dtype, vocab, dim, tokens, scale, ids_type):
    gen = torch.Generator().manual_seed(vocab + tokens)
    weight = torch.randn(vocab, dim, generator=gen).to(dtype)
    ids = draw_ids(tokens, vocab, "uniform", gen).to(ids_type)
    table = micro.TokenTable(vocab, dim, tokens, dtype=dtype)
    got = table.lookup(weight.to(DEV), ids.to(DEV), scale=scale)
    want = (weight[ids.long()].float() * torch.tensor(scale, dtype=torch.float32)).to(dtype)
    assert got.dtype == dtype and torch.equal(got.cpu(), want)


def test_lookup_of_strided_rows_and_shapes():
    gen = torch.Generator().manual_seed(1)
    base = torch.randn(40, 100, generator=gen).bfloat16().to(DEV)
    weight = base[:, 3:80]  # rows that start anywhere
    ids = torch.randint(0, 40, (4, 6), generator=gen).to(DEV)
    table = micro.TokenTable(40, 77, 24, dtype=torch.bfloat16)
    got = table.lookup(weight, ids)
    assert got.shape == (4, 6, 77) and torch.equal(got, weight[ids])
    out = torch.zeros(24, 91, dtype=torch.bfloat16, device=DEV)
    table.lookup(weight, ids, out=out[:, 5:82])
    assert torch.equal(out[:, 5:82], weight[ids.flatten()])
    assert bool((out[:, :5] == 0).all()) and bool((out[:, 82:] == 0).all())


def test_lookup_of_ids_outside_the_table_and_values_that_are_not_finite():
    weight = torch.tensor([[1.0, float("inf")], [float("nan"), -2.0]], device=DEV)
    table = micro.TokenTable(2, 2, 6)
    ids = torch.tensor([0, -1, 1, 2, 2 ** 40, -2 ** 40], device=DEV)
    got = table.lookup(weight, ids, scale=3.0).cpu()
    assert got[0].tolist() == [3.0, float("inf")]
    assert bool(got[2, 0].isnan()) and float(got[2, 1]) == -6.0
    assert bool(got[[1, 3, 4, 5]].isnan().all())


def test_lookup_past_32_bit_offsets():
    dim, vocab = 16384, 140_000  # 2.3e9 values
    weight = torch.zeros(vocab, dim, dtype=torch.bfloat16, device=DEV)
    weight[-1] = 3.0
    weight[vocab - 5, 7] = 5.0
    table = micro.TokenTable(vocab, dim, 4, dtype=torch.bfloat16)
    got = table.lookup(weight, torch.tensor([vocab - 1, 0, vocab - 5], device=DEV))
    assert bool((got[0] == 3.0).all()) and bool((got[1] == 0.0).all()) and float(got[2, 7]) == 5.0
    grad = torch.ones(4, dim, dtype=torch.bfloat16, device=DEV)
    table.lookup_grad(grad, torch.tensor([vocab - 1, 0, vocab - 1, 3], device=DEV), weight)
    assert bool((weight[-1] == 2.0).all()) and bool((weight[0] == 1.0).all()) and float(weight[vocab - 5].sum()) == 0.0
    assert float(weight.sum(dtype=torch.float64)) == 4.0 * dim


GRAD_CASES = [(1, 1, 1, "uniform"), (5, 3, 2, "uniform"), (10, 64, 31, "one"), (10, 64, 32, "one"), (10, 64, 33, "one"),
              (300, 77, 1000, "skewed"), (257, 128, 4097, "skewed"), (70_000, 16, 5000, "uniform"), (3, 40, 20_000, "one"),
              (1000, 24, 16_384, "skewed"), (1000, 24, 16_385, "skewed"), (65_537, 8, 70_001, "skewed"),
              (200, 2056, 300, "skewed"), (5000, 4, 4096, "skewed"), (5000, 4, 4097, "uniform"), (900, 4, 32_769, "skewed"),
              (70_000, 3, 300_001, "skewed"), (100, 64, 47, "one"), (100, 64, 48, "one"), (100, 64, 49, "one")]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("vocab,dim,tokens,kind", GRAD_CASES)
def test_lookup_grad(dtype, accumulate, vocab, dim, tokens, kind):
    gen = torch.Generator().manual_seed(vocab * 7 + tokens)
    ids = draw_ids(tokens, vocab, kind, gen)
    grad = torch.randn(tokens, dim, generator=gen).to(dtype)
    old = torch.randn(vocab, dim, generator=gen).to(dtype)
    table = micro.TokenTable(vocab, dim, tokens, dtype=dtype)
    dweight = old.to(DEV)
    got = table.lookup_grad(grad.to(DEV), ids.to(DEV), dweight, scale=1.5, accumulate=accumulate)
    assert got is dweight
    want, bound = ref.lookup_grad(grad, ids, vocab, 1.5, old if accumulate else None)
    assert ref.excess(got, want, bound) <= 1.0
    if accumulate:  # rows without a token are untouched, bit for bit
        absent = torch.bincount(ids, minlength=vocab) == 0
        assert torch.equal(got.cpu()[absent], old[absent])
    again = old.to(DEV)
    table.lookup_grad(grad.to(DEV), ids.to(DEV), again, scale=1.5, accumulate=accumulate)
    assert torch.equal(got.view(torch.uint8), again.view(torch.uint8))


def test_lookup_grad_is_the_derivative():
    """L = sum(out * d): the lookup is linear, so a central difference of L is
    exact up to rounding (in 64 bits, 1e-9)."""
    gen = torch.Generator().manual_seed(5)
    vocab, dim, tokens = 11, 6, 40
    ids = torch.randint(0, vocab, (tokens,), generator=gen)
    d = torch.randn(tokens, dim, generator=gen)
    table = micro.TokenTable(vocab, dim, tokens)
    got = table.lookup_grad(d.to(DEV), ids.to(DEV), torch.empty(vocab, dim, device=DEV), scale=0.5).cpu().double()
    w, step = torch.randn(vocab, dim, generator=gen).double(), torch.randn(vocab, dim, generator=gen).double()
    value = lambda x: float((0.5 * x[ids] * d.double()).sum())  # noqa: E731
    slope = (value(w + 1e-3 * step) - value(w - 1e-3 * step)) / 2e-3
    assert abs(slope - float((got * step).sum())) <= 1e-5 * float((got.abs() * step.abs()).sum())


def test_ids_that_have_no_part():
    vocab, dim = 20, 12
    ids = torch.tensor([3, -1, 20, 3, 2 ** 40, 5, 7], dtype=torch.int64)
    grad = torch.randn(7, dim, generator=torch.Generator().manual_seed(0))
    table = micro.TokenTable(vocab, dim, 7, padding_id=5)
    out = torch.full((vocab, dim), 9.0, device=DEV)
    table.lookup_grad(grad.to(DEV), ids.to(DEV), out)
    want, bound = ref.lookup_grad(grad, ids, vocab, 1.0, None, padding=5)
    assert ref.excess(out, want, bound) <= 1.0
    assert bool((out[5] == 0).all())
    table.lookup_grad(grad.to(DEV), torch.full((7,), 5, device=DEV), out, accumulate=True)
    assert ref.excess(out, want, bound) <= 1.0


def test_no_tokens():
    table = micro.TokenTable(5, 4, 0)
    ids = torch.empty(0, dtype=torch.int64, device=DEV)
    assert table.lookup(torch.ones(5, 4, device=DEV), ids).shape == (0, 4)
    out = torch.ones(5, 4, device=DEV)
    table.lookup_grad(torch.empty(0, 4, device=DEV), ids, out, accumulate=True)
    assert bool((out == 1).all())
    table.lookup_grad(torch.empty(0, 4, device=DEV), ids, out)
    assert bool((out == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("accumulate", [False, True])
def test_lookup_grad_of_strided_rows(dtype, accumulate):
    gen = torch.Generator().manual_seed(2)
    grad = torch.randn(90, 60, generator=gen).to(dtype)
    base = torch.full((30, 50), 4.0, dtype=dtype, device=DEV)
    ids = torch.randint(0, 29, (90,), generator=gen)
    table = micro.TokenTable(30, 37, 90, dtype=dtype)
    table.lookup_grad(grad.to(DEV)[:, 9:46], ids.to(DEV), base[:, 5:42], accumulate=accumulate)
    want, bound = ref.lookup_grad(grad[:, 9:46], ids, 30, 1.0, torch.full((30, 37), 4.0, dtype=dtype) if accumulate else None)
    assert ref.excess(base[:, 5:42], want, bound) <= 1.0
    assert bool((base[:, :5] == 4.0).all()) and bool((base[:, 42:] == 4.0).all())


def test_a_calls_of_different_lengths_on_one_handle():
    gen = torch.Generator().manual_seed(3)
    table = micro.TokenTable(500, 32, 40_000, dtype=torch.float32)
    for tokens in (40_000, 3, 17_000, 1, 0, 33_000):
        ids = draw_ids(tokens, 500, "skewed", gen) if tokens else torch.empty(0, dtype=torch.int64)
        grad = torch.randn(tokens, 32, generator=gen)
        out = torch.full((500, 32), 3.0, device=DEV)
        table.lookup_grad(grad.to(DEV), ids.to(DEV), out)
        want, bound = ref.lookup_grad(grad, ids, 500, 1.0, None)
        assert ref.excess(out, want, bound) <= 1.0


@pytest.mark.parametrize("tokens", [63, 64, 65, 1023, 4095, 8192, 8193, 65_536, 65_537, 66_600])
@pytest.mark.parametrize("kind", ["uniform", "skewed", "one"])
def test_order_of_tokens_around_the_sizes_of_its_steps(tokens, kind):
    """Ids outside the vocabulary and the padding id among the others: each row's
    terms are added once, the others nowhere."""
    gen = torch.Generator().manual_seed(tokens)
    ids = draw_ids(tokens, 700, kind, gen)
    ids[torch.rand(tokens, generator=gen) < 0.1] = 5
    outside = ids.clone()
    out = torch.rand(tokens, generator=gen) < 0.1
    outside[out] = torch.where(torch.rand(tokens, generator=gen) < 0.5, -1, 700)[out]
    grad = torch.randn(tokens, 12, generator=gen)
    table = micro.TokenTable(700, 12, tokens, padding_id=5)
    got = table.lookup_grad(grad.to(DEV), outside.to(DEV), torch.full((700, 12), 3.0, device=DEV))
    grad[out | (ids == 5)] = 0
    want, bound = ref.lookup_grad(grad, ids, 700, 1.0, None)
    assert ref.excess(got, want, bound) <= 1.0
    assert bool((got[5] == 0).all())


def test_refusals():
    weight = torch.ones(10, 8, device=DEV)
    table = micro.TokenTable(10, 8, 4)
    ids = torch.zeros(4, dtype=torch.int64, device=DEV)
    out = torch.full((4, 8), 7.0, device=DEV)
    bad = [lambda: table.lookup(weight, ids.float()), lambda: table.lookup(weight, ids.cpu()),
           lambda: table.lookup(weight[:9], ids), lambda: table.lookup(weight.half(), ids),
           lambda: table.lookup(weight, torch.zeros(5, dtype=torch.int64, device=DEV)),
           lambda: table.lookup(weight, ids, out=out[:3]), lambda: table.lookup(weight, ids, out=weight[:4]),
           lambda: table.lookup(weight.t().contiguous().t(), ids), lambda: table.lookup(weight, ids[::2]),
           lambda: table.lookup_grad(out, ids, weight[:, :4]), lambda: table.lookup_grad(out, ids, out),
           lambda: table.lookup_grad(out[:3], ids, weight), lambda: table.lookup_grad(weight[:4], ids, weight)]
    for call in bad:
        with pytest.raises((TypeError, ValueError, _lib.MicroError)):
            call()
    torch.cuda.synchronize()
    assert bool((weight == 1).all()) and bool((out == 7).all())
    with pytest.raises(_lib.MicroError) as e:
        table.lookup(weight, torch.zeros(5, dtype=torch.int64, device=DEV))
    assert e.value.status == _lib.MICRO_ECAPACITY
    for args, status in (((0, 8, 4), _lib.MICRO_EINVAL), ((10, 0, 4), _lib.MICRO_EINVAL), ((10, 8, -1), _lib.MICRO_EINVAL),
                         ((2 ** 31, 8, 4), _lib.MICRO_ERANGE), ((10, 65537, 4), _lib.MICRO_ERANGE),
                         ((10, 8, 2 ** 22 + 1), _lib.MICRO_ERANGE)):
        with pytest.raises(_lib.MicroError) as e:
            micro.TokenTable(*args)
        assert e.value.status == status
    with pytest.raises(TypeError):
        micro.TokenTable(10, 8, 4, dtype=torch.float64)
    table.close()
    with pytest.raises(RuntimeError):
        table.lookup(weight, ids)


def test_another_stream():
    stream = torch.cuda.Stream()
    table = micro.TokenTable(100, 64, 50, stream=stream)
    weight = torch.randn(100, 64, device=DEV)
    ids = torch.randint(0, 100, (50,), device=DEV)
    torch.cuda.synchronize()
    got = table.lookup(weight, ids)
    stream.synchronize()
    assert torch.equal(got, weight[ids])
