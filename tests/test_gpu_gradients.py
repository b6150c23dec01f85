"""The gradient set on the GPU: the global norm, clipping in place and into the
flat vector, against the definition in 64 bits."""
import ctypes
import math

import pytest
import torch

import paper_2310_00967_amd as micro
from paper_2310_00967_amd import _lib

from language_reference import EPS, TINY, U

pytestmark = pytest.mark.gpu

DEV = "cuda"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def make(sizes, types, seed=0, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn(n, generator=gen).mul_(scale).to(t).to(DEV) for n, t in zip(sizes, types)]


def definition(tensors, max_norm, sumsq=None):
    """(norm, factor, scaled values per tensor) in 64 bits."""
    host = [t.cpu().double() for t in tensors]
    square = math.fsum(float((x * x).sum()) for x in host) if sumsq is None else sumsq
    norm = math.sqrt(square)
    c = min(1.0, max_norm / (norm + 1e-6)) if max_norm != math.inf else 1.0
    return norm, c, [x * c for x in host]


SETS = [
    ([1], [F32]), ([1], [BF16]), ([5, 0, 3], [F16, F32, BF16]), ([2048], [F32]), ([4095, 4096, 4097], [F32, BF16, F16]),
    ([100_003, 7, 65_536, 1], [BF16, F32, BF16, F16]), ([3_000_001], [BF16]), ([1_234_567, 2_345_678], [F16, F32]),
    ([33] * 300, [BF16, F32, F16] * 100), ([20_000_003, 5, 9_999_999], [BF16, F32, F32]),
]


@pytest.mark.parametrize("sizes,types", SETS)
@pytest.mark.parametrize("max_norm", [0.25, 1e9])
def test_norm_flatten_and_clip(sizes, types, max_norm):
    tensors = make(sizes, types)
    grads = micro.GradientSet(tensors)
    norm, c, want = definition(tensors, max_norm)
    # binary64 products are exact, sums within (n - 1) 2^-53
    assert abs(float(grads.sumsq()) - norm * norm) <= (sum(sizes) + 8) * 2.0 ** -53 * norm * norm
    assert abs(float(grads.norm()) - norm) <= 2 * EPS * norm
    flat = torch.full((sum(sizes) + 2,), -7.0, device=DEV)
    got = grads.flatten(flat[1:-1], max_norm=max_norm)
    assert got.dtype == F32 and got.shape == ()
    assert abs(float(got) - norm) <= 2 * EPS * norm
    # the factor's rounding and the product's
    f = flat.cpu().double()
    assert float(f[0]) == -7.0 and float(f[-1]) == -7.0
    w = torch.cat(want)
    assert bool(((f[1:-1] - w).abs() <= 3 * EPS * w.abs() + TINY[F32]).all())
    if c == 1.0:
        assert torch.equal(flat[1:-1], torch.cat([t.float() for t in tensors]))
    for t, x in zip(tensors, definition(tensors, math.inf)[2]):
        assert torch.equal(t.cpu().double(), x)  # flatten leaves the tensors alone
    assert abs(float(grads.clip_(max_norm)) - norm) <= 2 * EPS * norm
    for t, x in zip(tensors, want):
        u = U[t.dtype] + (3 * EPS if c != 1.0 else 0.0)
        assert bool(((t.cpu().double() - x).abs() <= u * x.abs() * 1.01 + TINY[t.dtype]).all()), t.dtype
    grads.close()


def test_results_do_not_change_between_runs():
    tensors = make([3_000_017, 1_000_003], [F32, BF16])
    grads = micro.GradientSet(tensors)
    first = grads.sumsq().clone()
    for _ in range(20):
        assert torch.equal(grads.sumsq(), first)


def test_conversion_without_a_norm():
    tensors = make([1000, 77], [BF16, F32])
    tensors[0][3] = math.inf
    tensors[1][5] = math.nan
    grads = micro.GradientSet(tensors)
    flat = torch.empty(1077, device=DEV)
    assert grads.flatten(flat) is None
    assert torch.equal(flat.view(torch.int32), torch.cat([t.float() for t in tensors]).view(torch.int32))
    norm = grads.flatten(flat, max_norm=math.inf)
    assert math.isnan(float(norm))
    assert torch.equal(flat.view(torch.int32), torch.cat([t.float() for t in tensors]).view(torch.int32))


def test_another_workers_sum():
    tensors = make([5000, 70], [F32, BF16])
    grads = micro.GradientSet(tensors)
    total = grads.sumsq() * 4.0
    norm, c, want = definition(tensors, 1.0, float(total))
    flat = torch.empty(5070, device=DEV)
    assert abs(float(grads.flatten(flat, max_norm=1.0, sumsq=total)) - norm) <= 2 * EPS * norm
    w = torch.cat(want)
    assert bool(((flat.cpu().double() - w).abs() <= 3 * EPS * w.abs()).all())
    assert abs(float(grads.clip_(1.0, sumsq=total)) - norm) <= 2 * EPS * norm
    assert bool(((tensors[0].cpu().double() - want[0]).abs() <= 3 * EPS * want[0].abs()).all())


def test_values_whose_squares_leave_binary32():
    tensors = [torch.tensor([3e38, -3e38], device=DEV), torch.tensor([1e-38] * 5, device=DEV)]
    grads = micro.GradientSet(tensors)
    want = math.sqrt(float(sum((t.double() ** 2).sum() for t in tensors)))
    assert abs(float(grads.sumsq()) - want * want) <= 1e-14 * want * want
    small = micro.GradientSet(tensors[1:])
    assert abs(float(small.norm()) / (1e-38 * math.sqrt(5)) - 1) < 1e-6


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_value_that_is_not_finite(bad):
    """The formula: a norm of +inf gives the factor 0 (and 0 * inf = NaN), a
    NaN makes everything NaN."""
    tensors = make([300, 40], [F32, BF16])
    tensors[0][17] = bad
    grads = micro.GradientSet(tensors)
    flat = torch.empty(340, device=DEV)
    norm = float(grads.flatten(flat, max_norm=1.0))
    if math.isnan(bad):
        assert math.isnan(norm) and bool(flat.isnan().all())
    else:
        assert norm == math.inf and bool(flat[17].isnan())
        flat[17] = 0.0
        assert bool((flat == 0.0).all())


@pytest.mark.parametrize("offset", [1, 2, 3, 5])
def test_tensors_and_vectors_that_start_anywhere(offset):
    base = make([5000 + offset, 9000 + offset], [BF16, F32], seed=3)
    tensors = [base[0][offset:], base[1][offset:]]
    grads = micro.GradientSet(tensors)
    norm, c, want = definition(tensors, 2.0)
    flat = torch.empty(14_000 + offset, device=DEV)[offset:]
    assert abs(float(grads.flatten(flat, max_norm=2.0)) - norm) <= 2 * EPS * norm
    w = torch.cat(want)
    assert bool(((flat.cpu().double() - w).abs() <= 3 * EPS * w.abs()).all())
    before = [base[0][:offset].clone(), base[1][:offset].clone()]
    grads.clip_(2.0)
    assert torch.equal(base[0][:offset], before[0]) and torch.equal(base[1][:offset], before[1])


def test_no_values():
    for tensors in ([], [torch.empty(0, device=DEV)]):
        grads = micro.GradientSet(tensors, device=DEV)
        assert float(grads.norm()) == 0.0
        assert float(grads.clip_(1.0)) == 0.0
        assert float(grads.flatten(torch.empty(0, device=DEV), max_norm=1.0)) == 0.0


def test_another_stream():
    stream = torch.cuda.Stream()
    tensors = make([200_003], [F32])
    torch.cuda.synchronize()
    grads = micro.GradientSet(tensors, stream=stream)
    flat = torch.empty(200_003, device=DEV)
    norm = grads.flatten(flat, max_norm=0.5)
    stream.synchronize()
    want, c, values = definition(tensors, 0.5)
    assert abs(float(norm) - want) <= 2 * EPS * want
    assert bool(((flat.cpu().double() - values[0]).abs() <= 3 * EPS * values[0].abs()).all())


def test_a_graph_replays():
    tensors = make([100_003, 50], [F32, BF16])
    stream = torch.cuda.Stream()
    grads = micro.GradientSet(tensors, stream=stream)
    flat = torch.empty(100_053, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        grads.flatten(flat, max_norm=1.0)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            norm = grads.flatten(flat, max_norm=1.0)
    for seed in range(4):
        for t, x in zip(tensors, make([100_003, 50], [F32, BF16], seed=seed, scale=seed + 0.5)):
            t.copy_(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, c, values = definition(tensors, 1.0)
        assert abs(float(norm) - want) <= 2 * EPS * want
        w = torch.cat(values)
        assert bool(((flat.cpu().double() - w).abs() <= 3 * EPS * w.abs()).all())
        torch.cuda.synchronize()


def test_refusals():
    a, b = make([100, 50], [F32, BF16])
    for tensors in ([a, a], [a, a[10:20]], [a.view(10, 10).t()], [a.double()], [a.cpu()], [3.0]):
        with pytest.raises((TypeError, _lib.MicroError)):
            micro.GradientSet(tensors, device=DEV)
    grads = micro.GradientSet([a, b])
    flat = torch.full((150,), 5.0, device=DEV)
    keep = (a.clone(), b.clone())
    for call in (lambda: grads.flatten(flat[:149]), lambda: grads.flatten(flat.double()),
                 lambda: grads.flatten(torch.empty(300, device=DEV)[::2]), lambda: grads.flatten(flat, sumsq=flat[:1].double()),
                 lambda: grads.flatten(flat, max_norm=1.0, sumsq=flat[:1]), lambda: grads.clip_(0.0),
                 lambda: grads.clip_(math.nan), lambda: grads.clip_(-1.0), lambda: grads.flatten(flat, max_norm=0.0)):
        with pytest.raises((TypeError, ValueError, _lib.MicroError)):
            call()
    one = micro.GradientSet([flat])
    with pytest.raises(_lib.MicroError) as e:
        one.flatten(flat)
    assert e.value.status == _lib.MICRO_EINVAL and "memory" in str(e.value)
    torch.cuda.synchronize()
    assert torch.equal(a, keep[0]) and torch.equal(b, keep[1]) and bool((flat == 5.0).all())
    lib = _lib.load()
    assert lib.micro_grads_norm(grads._handle, None, None) == _lib.MICRO_EINVAL
    assert lib.micro_grads_norm(grads._handle, ctypes.c_void_p(a.data_ptr()), None) == _lib.MICRO_EINVAL
    assert lib.micro_grads_norm(grads._handle, ctypes.c_void_p(flat.data_ptr() + 4), None) == _lib.MICRO_EINVAL
    grads.close()
    grads.close()
    with pytest.raises(RuntimeError):
        grads.norm()
