"""The token table's kernels where their workgroups take more than one tile, and
where the order of tokens takes all four digits, against the same definitions
and bounds as the smaller cases."""
import pytest
import torch

import paper_2310_00967_amd as micro

import language_reference as ref
from test_gpu_loss import check, make

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,dim,tokens,counted", [
    (24_100, 192, 700, 1.0),   # 95 x 3 wide tiles of scores on 256 workgroups, three steps each
    (24_100, 200, 1500, 0.4),  # some of them without a token; a padded width
    (33_000, 192, 300, 1.0),   # 258 x 3 middle tiles on 512
    (300, 2100, 8200, 1.0),    # 9 x 33 wide tiles of dhidden
    (40, 22_000, 384, 1.0),    # 172 x 3 middle tiles of dhidden
])
def test_more_tiles_than_workgroups(dtype, vocab, dim, tokens, counted):
    table = micro.TokenTable(vocab, dim, tokens, dtype=dtype)
    check(table, *make(vocab, dim, tokens, dtype, counted=counted), scale=32.0)
    table.close()


@pytest.mark.parametrize("dtype", TYPES)
def test_the_loss_alone_of_few_tokens_over_many_rows(dtype):
    """1095 narrow tiles on 1024 workgroups."""
    hidden, weight, targets = make(140_100, 192, 20, dtype)
    targets[0], targets[1], targets[2] = 140_099, 131_071, 131_072  # the last tile, and both sides of the second round
    table = micro.TokenTable(140_100, 192, 20, dtype=dtype)
    loss, losses = table.loss(hidden.to(DEV), weight.to(DEV), targets.to(DEV))
    r = ref.loss(hidden, weight, targets, True)
    assert ref.excess(losses, r["losses"], r["error"] + 2 * ref.EPS * r["losses"].abs() + 1e-300) <= 1.0
    assert ref.excess(loss, r["loss"], r["error"].sum() / 20 + 2 * ref.EPS * r["loss"].abs()) <= 1.0


@pytest.mark.parametrize("tokens", [8000, 9000])  # counted order, sorted order
@pytest.mark.parametrize("accumulate", [False, True])
def test_a_vocabulary_of_four_digits(tokens, accumulate):
    vocab, dim = 2 ** 24 + 5, 2
    gen = torch.Generator().manual_seed(1)
    ids = torch.randint(2 ** 24 - 40, vocab, (tokens,), generator=gen)
    low = torch.rand(tokens, generator=gen) < 0.5
    ids[low] -= 2 ** 24 - 40  # the same last digits
    ids[torch.rand(tokens, generator=gen) < 0.05] = vocab  # outside
    grad = torch.randn(tokens, dim, generator=gen)
    old = torch.full((vocab, dim), 0.5)
    table = micro.TokenTable(vocab, dim, tokens)
    got = table.lookup_grad(grad.to(DEV), ids.to(DEV), old.to(DEV), scale=1.5, accumulate=accumulate)
    want, bound = ref.lookup_grad(grad, ids, vocab, 1.5, old if accumulate else None)
    assert ref.excess(got, want, bound) <= 1.0
