"""Draws of more rows than the card has compute units, which smaller workgroups with
shorter lists make: the same tokens as for few rows, against the definition in the same
way, in every type and under every kind of settings."""
import math

import pytest
import torch

import paper_2310_00967_amd as micro

import sample_reference as ref
import test_gpu_sample as few

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = few.TYPES


def units():
    return torch.cuda.get_device_properties(0).multi_processor_count


class Repeated:
    """The rows of every call, drawn again and again until there are `rows` of them (by
    default more than compute units): each repetition has to be answered alike, and the
    tokens are those of the few rows alone."""

    def __init__(self, vocab, rows=None):
        self.rows = rows or units() + 45
        self.table = micro.TokenTable(vocab, 1, self.rows)

    def sample(self, logits, uniforms, out=None, **settings):
        n = uniforms.numel()
        at = torch.arange(self.rows, device=DEV) % n
        many = {k: v[at].contiguous() if isinstance(v, torch.Tensor) else v for k, v in settings.items()}
        to = None if out is None else torch.empty(self.rows, dtype=out.dtype, device=DEV)
        ids, logprobs = self.table.sample(logits[at].contiguous(), uniforms[at].contiguous(), out=to, **many)
        bits = logprobs.view(torch.int32)
        assert torch.equal(ids, ids[:n][at]) and torch.equal(bits, bits[:n][at])
        alone = self.table.sample(logits, uniforms, **settings)
        assert torch.equal(ids[:n].long(), alone[0])
        return ids[:n], logprobs[:n]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("settings", few.SETTINGS, ids=lambda s: "-".join(f"{k}{v}" for k, v in s.items()) or "plain")
@pytest.mark.parametrize("rows,vocab", [(3, 1), (6, 63), (7, 1000), (5, 8193)])
def test_settings_of_all_rows(dtype, settings, rows, vocab):
    logits, uniforms = few.rows_of(rows, vocab, dtype, vocab + 1)
    few.check(Repeated(vocab), logits, uniforms, **settings)


@pytest.mark.parametrize("dtype", TYPES)
def test_settings_of_every_row(dtype):
    """Of top_k the ends of the lists of both workgroups among them, and what
    takes histograms."""
    rows, vocab = 60, 4099
    logits, uniforms = few.rows_of(rows, vocab, dtype, 15)
    gen = torch.Generator().manual_seed(18)
    pick = lambda v, t: torch.tensor(v, dtype=t)[torch.randint(len(v), (rows,), generator=gen)]  # noqa: E731
    few.check(Repeated(vocab), logits, uniforms, temperature=pick([0.0, 0.5, 1.0, 2.0], torch.float32),
              top_k=pick([0, 1, 7, 255, 256, 257, 300, 511, 512, 513, 1024, 1025, 4098, 4099, 5000], torch.int32),
              top_p=pick([1.0, 0.5, 0.97], torch.float32), min_p=pick([0.0, 0.02, 0.5], torch.float32))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("settings", [{}, {"top_p": 0.97}, {"min_p": 0.01}], ids=["", "top_p", "min_p"])
@pytest.mark.parametrize("top_k", [255, 256, 257, 511, 512, 513, 1024])
def test_top_k_at_the_ends_of_the_lists(dtype, settings, top_k):
    vocab = 5003
    logits, uniforms = few.rows_of(8, vocab, dtype, top_k)
    few.check(Repeated(vocab), logits, uniforms, temperature=1.7, top_k=top_k, **settings)
    each = torch.full((8,), top_k, dtype=torch.int32)
    few.check(Repeated(vocab), logits, uniforms, temperature=1.7, top_k=each, **settings)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("settings", [{}, {"top_k": 20}, {"top_p": 0.5}, {"top_k": 30, "top_p": 0.5}, {"min_p": 0.9},
                                      {"temperature": 0.0}, {"top_k": 300}, {"top_k": 700, "top_p": 0.9}])
def test_many_equal_logits(dtype, settings):
    """Cuts that fall among as many equal logits as either workgroup's list holds, and
    one more or less."""
    vocab = 5001
    counts = [255, 256, 257, 511, 512, 513, 800, 1023, 1024, 1025]
    gen = torch.Generator().manual_seed(6)
    logits = torch.full((len(counts) + 2, vocab), -30.0)
    for r, n in enumerate(counts):
        logits[r, torch.randperm(vocab, generator=gen)[:n]] = 1.0
        logits[r, torch.randint(vocab, (3,), generator=gen)] = 2.0
    logits[-2] = 0.0
    logits[-1] = torch.randint(0, 4, (vocab,), generator=gen).float()
    few.check(Repeated(vocab), logits.to(dtype), torch.rand(len(logits), generator=gen), **settings)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("settings", [{}, {"top_k": 5}, {"top_p": 0.8}, {"temperature": 0.0}, {"min_p": 0.1},
                                      {"top_k": 400, "top_p": 0.9}, {"temperature": math.inf}])
def test_masked_rows_and_values_that_are_not_finite(dtype, settings):
    vocab, inf = 777, math.inf
    logits, uniforms = few.rows_of(10, vocab, dtype, 12)
    logits[0] = -inf
    logits[1] = math.nan
    logits[2] = -inf
    logits[2, vocab - 1] = -5.0
    logits[3, ::2] = -inf
    logits[4, 1::2] = math.nan
    logits[5, [3, 70, 500]] = inf
    logits[6, 0] = inf
    logits[7, 100:] = torch.finfo(dtype).min
    logits[8] = torch.finfo(dtype).min
    logits[9, 5] = torch.finfo(dtype).max
    ids, _ = few.check(Repeated(vocab), logits, uniforms, **settings)
    assert ids[:3].tolist() == [-1, -1, vocab - 1] and int(ids[6]) == 0


def test_uniforms_at_the_ends():
    vocab = 1000
    logits, _ = few.rows_of(1, vocab, torch.float32, 4)
    logits[0, :10] = -math.inf
    logits[0, 990:] = -math.inf
    u = torch.tensor([0.0, -1.0, math.nan, 1.0, 2.0, math.inf, 1.0 - 2.0 ** -24, 2.0 ** -149])
    for settings in ({}, {"top_k": 990}, {"top_p": 1.0 - 2.0 ** -30}):
        ids, _ = few.check(Repeated(vocab), logits.expand(u.numel(), vocab).contiguous(), u, **settings)
        assert ids[:3].tolist() == [10, 10, 10] and ids[3:6].tolist() == [989, 989, 989]


@pytest.mark.parametrize("more", [-1, 0, 1])
def test_as_many_rows_as_compute_units(more):
    vocab = 600
    logits, uniforms = few.rows_of(13, vocab, torch.bfloat16, 31)
    for settings in ({"top_p": 0.9}, {"top_k": 300}, {"top_k": 20, "min_p": 0.05}):
        few.check(Repeated(vocab, units() + more), logits, uniforms, out=torch.empty(1, dtype=torch.int32), **settings)


def test_strided_rows():
    vocab, rows = 1031, units() + 9
    logits, uniforms = few.rows_of(rows, vocab, torch.float16, 9)
    table = micro.TokenTable(vocab, 1, rows)
    base = torch.zeros(rows, vocab + 100, dtype=torch.float16, device=DEV)
    base[:, 33:33 + vocab] = logits.to(DEV)
    for settings in ({}, {"top_p": 0.9}, {"top_k": 40}, {"top_k": 400}, {"temperature": 0.0}):
        want = table.sample(logits.to(DEV), uniforms.to(DEV), **settings)
        got = table.sample(base[:, 33:33 + vocab], uniforms.to(DEV), **settings)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        for r in (0, rows // 2, rows - 1):
            tokens, _ = ref.draw(logits[r].double().numpy(), float(uniforms[r]), **settings)
            assert int(want[0][r]) in tokens
