"""Packing into microscaled 4-bit matrices and their products on the GPU, against
their definitions: codes, scales and unpacked values bit for bit, products within
their derived bound."""
import pytest
import torch

import paper_2310_00967_amd as micro

import language_reference
import microscaled_reference as ref
from test_microscaled_abi import changes_in_place

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def draw(rows, cols, dtype, seed):
    """Values whose blocks' sizes span many powers of two."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=gen)
    return (x * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=gen).float()
                           + torch.randint(-4, 4, (1, cols), generator=gen).float())).to(dtype)


def check_packed(got, x):
    code, scale = ref.quantise(x)
    codes, scales = ref.layout(code, scale)
    assert got.shape == tuple(x.shape)
    assert torch.equal(got.scales.cpu(), scales)
    assert torch.equal(got.codes.cpu(), codes)


SIZES = [(1, 1), (1, 32), (3, 31), (16, 33), (5, 255), (33, 256), (37, 257), (300, 77), (64, 1024), (129, 2085), (700, 64),
         (2, 5000), (257, 300)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_pack(dtype, rows, cols):
    x = draw(rows, cols, dtype, rows * 31 + cols)
    mx = micro.Microscaled()
    check_packed(mx.pack(x.to(DEV)), x)
    check_packed(mx.pack(x.to(DEV), transposed=True), x.t())
    q, t = mx.pack_both(x.to(DEV))
    check_packed(q, x)
    check_packed(t, x.t())


@pytest.mark.parametrize("dtype", TYPES)
def test_pack_every_rounding(dtype):
    """Every level, every border between two levels and the values next to both,
    under scales from the least to the largest."""
    levels = [0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.0, 7.75]
    points = torch.tensor(levels, dtype=torch.float64).to(dtype)
    near = torch.cat([points, torch.nextafter(points, points + 1), torch.nextafter(points, points - 1)])
    near = near[near < 8].float()
    near = torch.cat([near, -near])
    low, high = {torch.float32: (-149, 126), torch.float16: (-26, 13), torch.bfloat16: (-135, 126)}[dtype]
    rows = []
    for e in range(low, high):
        for at in range(0, near.numel(), 31):
            part = near[at:at + 31]
            rows.append(torch.cat([torch.tensor([4.0]), part, torch.zeros(31 - part.numel())]).double() * 2.0 ** e)
    x = torch.stack(rows).to(dtype)
    x = x[x.isfinite().all(1)]
    mx = micro.Microscaled()
    check_packed(mx.pack(x.to(DEV)), x)
    check_packed(mx.pack(x.t().contiguous().to(DEV), transposed=True), x)


@pytest.mark.parametrize("dtype", TYPES)
def test_pack_of_values_that_are_not_finite_and_zeros(dtype):
    x = draw(9, 300, dtype, 4)
    x[0, 40], x[1, 299], x[2, 0] = float("nan"), float("inf"), -float("inf")
    x[3], x[4, :32], x[5, 64:96] = 0.0, 0.0, -0.0
    x[6], x[7, :40] = torch.finfo(dtype).max, torch.finfo(dtype).tiny
    x[8, :32] = ref.TINY[dtype]
    mx = micro.Microscaled()
    for got, want in ((mx.pack(x.to(DEV)), x), (mx.pack(x.to(DEV), transposed=True), x.t())):
        check_packed(got, want)
        back = mx.unpack(got).cpu().double()
        exact = ref.packed_values(want)
        assert torch.equal(back.isnan(), exact.isnan())
        assert torch.equal(back.nan_to_num(), exact.nan_to_num())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (37, 257), (64, 1024), (129, 2085)])
def test_unpack(dtype, rows, cols):
    x = draw(rows, cols, torch.float32, cols)
    mx = micro.Microscaled()
    q = mx.pack(x.to(DEV))
    want = ref.packed_values(x)
    got = mx.unpack(q, dtype)
    assert got.dtype == dtype and torch.equal(got.cpu(), want.to(dtype))
    out = torch.full((rows, cols + 11), 5.0, dtype=dtype, device=DEV)
    assert mx.unpack(q, out=out[:, 3:3 + cols]).data_ptr() == out[:, 3:].data_ptr()
    assert torch.equal(out[:, 3:3 + cols].cpu(), want.to(dtype))
    assert bool((out[:, :3] == 5).all()) and bool((out[:, 3 + cols:] == 5).all())


def test_strided_rows_and_shapes():
    base = draw(40, 600, torch.bfloat16, 1).to(DEV)
    mx = micro.Microscaled()
    x = base[:, 5:505]
    check_packed(mx.pack(x), x.cpu())
    check_packed(mx.pack(x, transposed=True), x.cpu().t())
    check_packed(mx.pack(base.view(4, 10, 600)), base.cpu())
    w = mx.pack(draw(24, 600, torch.bfloat16, 2).to(DEV))
    y = mx.linear(base.view(4, 10, 600), w)
    assert y.shape == (4, 10, 24) and torch.equal(y.view(40, 24), mx.linear(base, w))
    assert mx.linear(base[0], w).shape == (24,)


PRODUCTS = [(1, 1, 1), (1, 5, 33), (1, 1000, 2048), (2, 31, 256), (7, 300, 77), (19, 129, 300), (32, 64, 1025), (33, 65, 512),
            (64, 64, 64), (100, 257, 130), (130, 1000, 511), (257, 255, 256), (300, 520, 700), (1000, 90, 2304),
            (520, 1030, 40), (40, 37, 9000), (1024, 768, 1280)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(dtype, m, n, k):
    a, b = draw(m, k, torch.bfloat16, m + k), draw(n, k, torch.bfloat16, n + 7 * k)
    if dtype == torch.float16:  # within its range
        a, b = a / 2.0 ** 9, b / 2.0 ** 9
    mx = micro.Microscaled()
    qa, qb = mx.pack(a.to(DEV)), mx.pack(b.to(DEV))
    got = mx.product(qa, qb, dtype=dtype)
    va, vb = ref.packed_values(a), ref.packed_values(b)
    want, bound = ref.product(va, vb, dtype)
    assert got.dtype == dtype and language_reference.excess(got, want, bound) <= 1.0
    assert torch.equal(got, mx.product(qa, qb, dtype=dtype))
    assert torch.equal(got, mx.linear(a.to(DEV), qb, dtype=dtype))
    # into strided rows, added to what is there
    old = torch.randn(m, n, generator=torch.Generator().manual_seed(m)).to(dtype)
    whole = torch.full((m, n + 9), 3.0, dtype=dtype, device=DEV)
    out = whole[:, 5:5 + n]
    out.copy_(old)
    assert mx.product(qa, qb, out=out, accumulate=True) is out
    want, bound = ref.product(va, vb, dtype, old)
    assert language_reference.excess(out, want, bound) <= 1.0
    assert bool((whole[:, :5] == 3).all()) and bool((whole[:, 5 + n:] == 3).all())


@pytest.mark.parametrize("x_type", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 70, 2048), (4, 300, 2041), (5, 33, 1500), (32, 100, 256), (31, 40, 129),
                                   (33, 40, 100), (1, 40, 8192), (1, 40, 8193), (2, 1, 4096)])
def test_linear_of_few_rows(x_type, dtype, m, n, k):
    """Rows that the workgroups pack themselves (up to 32 of 8192 values in whole groups
    together) and more: as what is packed first."""
    base = draw(m, k + 6, x_type, m + k).to(DEV)
    base = base / 2.0 ** 9
    x = base[:, 3:3 + k]
    w = draw(n, k, torch.float32, n) / 2.0 ** 9
    mx = micro.Microscaled()
    q, qx = mx.pack(w.to(DEV)), mx.pack(x)
    check_packed(qx, x.cpu())
    got = mx.linear(x, q, dtype=dtype)
    want, bound = ref.product(ref.packed_values(x.cpu()), ref.packed_values(w), dtype)
    assert got.dtype == dtype and language_reference.excess(got, want, bound) <= 1.0
    assert torch.equal(got, mx.product(qx, q, dtype=dtype))
    whole = torch.full((m, n + 9), 3.0, dtype=dtype, device=DEV)
    mx.linear(x, q, out=whole[:, 5:5 + n], accumulate=True)
    want, bound = ref.product(ref.packed_values(x.cpu()), ref.packed_values(w), dtype, torch.full((m, n), 3.0))
    assert language_reference.excess(whole[:, 5:5 + n], want, bound) <= 1.0
    assert bool((whole[:, :5] == 3).all()) and bool((whole[:, 5 + n:] == 3).all())
    x[0, k // 2] = float("nan")
    got = mx.linear(x, q, dtype=dtype)
    assert bool(got[0].isnan().all()) and not bool(got[1:].isnan().any())


# (rows, columns, length): middle tiles in one round and in several, wide ones in one and
# in two, each with an odd number of groups, edges on both sides and a tail cut along the sum
LARGE_PRODUCTS = [(2000, 2300, 130), (1500, 3001, 300), (2000, 9000, 40), (2050, 9000, 257), (500, 1000, 9000),
                  (130, 5000, 8200), (250, 65500, 300), (256, 65536, 512), (500, 50000, 130), (4100, 4096, 640),
                  (256, 65600, 8300)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", LARGE_PRODUCTS)
def test_large_product(dtype, m, n, k):
    gen = torch.Generator(device=DEV).manual_seed(m + n + k)
    draw_on = lambda rows: torch.randn(rows, k, generator=gen, device=DEV) * torch.exp2(  # noqa: E731
        torch.randint(-3, 3, (rows, 1), generator=gen, device=DEV).float())
    mx = micro.Microscaled()
    qa, qb = mx.pack(draw_on(m)), mx.pack(draw_on(n))
    got = mx.product(qa, qb, dtype=dtype)
    rows = torch.unique(torch.cat([torch.arange(0, m, max(1, m // 60)), torch.tensor([0, m // 2, m - 1])])).to(DEV)
    va, vb = mx.unpack(qa).double()[rows], mx.unpack(qb).double()
    want, bound = ref.product(va, vb, dtype)
    assert float(((got[rows].double() - want).abs() / bound).max()) <= 1.0
    assert torch.equal(got, mx.product(qa, qb, dtype=dtype))
    # the other way around, every row against what was checked above
    assert float(((mx.product(qb, qa, dtype=dtype)[:, rows].t().double() - want).abs() / bound).max()) <= 1.0
    # into strided rows, added to what is there
    whole = torch.full((m, n + 9), 3.0, dtype=dtype, device=DEV)
    old = torch.randn(rows.numel(), n, generator=gen, device=DEV).to(dtype)
    whole[rows, 5:5 + n] = old
    out = whole[:, 5:5 + n]
    mx.product(qa, qb, out=out, accumulate=True)
    want, bound = ref.product(va, vb, dtype, old)
    assert float(((out[rows].double() - want).abs() / bound).max()) <= 1.0
    assert bool((whole[:, :5] == 3).all()) and bool((whole[:, 5 + n:] == 3).all())
    # rows that were not looked at are what the sum of one more row would be
    plain = mx.product(qa, qb, dtype=dtype)
    rest = torch.ones(m, dtype=torch.bool, device=DEV)
    rest[rows] = False
    want = plain[rest].double() + 3.0
    # one sum in binary32 and its rounding against two roundings to the type
    slack = (2 * ref.U[dtype] + 4 * ref.EPS) * (plain[rest].double().abs() + 3.0) * (1 + ref.U[dtype])
    assert bool(((out[rest].double() - want).abs() <= slack).all())


@pytest.mark.parametrize("m,n", [(3, 40), (100, 300), (2100, 2300), (250, 65540)])
def test_product_of_blocks_that_are_not_numbers(m, n):
    """A NaN block reaches its own row's and column's sums, whatever it meets."""
    a, b = torch.ones(m, 300), torch.ones(n, 300)
    a[1, 100], b[5, 299] = float("nan"), float("inf")
    b[:, 96:128] = 0.0
    mx = micro.Microscaled()
    got = mx.product(mx.pack(a.to(DEV)), mx.pack(b.to(DEV)))
    nan = torch.zeros(m, n, dtype=torch.bool, device=DEV)
    nan[1], nan[:, 5] = True, True
    assert torch.equal(got.isnan(), nan)


@pytest.mark.parametrize("m,n", [(2, 40), (60, 70), (2100, 2300), (250, 65540)])
def test_product_at_the_ends_of_the_range(m, n):
    """Blocks of the largest and the smallest scales: sums past binary32 are
    infinite, products below its least are lost, and nothing else is."""
    a, b = torch.ones(m, 64), torch.ones(n, 64)
    a[0], a[1, :32] = 2.0 ** 100, 2.0 ** -126
    b[0], b[1] = 2.0 ** 40, 2.0 ** -100
    b[2], b[3] = 2.0 ** 20, 2.0 ** 126
    a[1, 32:] = 0.0
    mx = micro.Microscaled()
    got = mx.product(mx.pack(a.to(DEV)), mx.pack(b.to(DEV))).cpu()
    assert float(got[0, 0]) == float("inf") and float(got[0, 1]) == 64.0 and float(got[0, 2]) == 2.0 ** 126
    assert float(got[1, 2]) == 2.0 ** -101 and float(got[1, 3]) == 32.0 and float(got[1, 0]) == 2.0 ** -81
    assert abs(float(got[1, 1])) <= 2.0 ** -149
    assert bool((got[2:, 4:] == 64.0).all())


def test_empty_sides():
    mx = micro.Microscaled()
    none = mx.pack(torch.empty(0, 40, device=DEV))
    some = mx.pack(torch.ones(7, 40, device=DEV))
    assert mx.product(none, some).shape == (0, 7) and mx.product(some, none).shape == (7, 0)
    flat = mx.pack(torch.empty(7, 0, device=DEV))
    assert flat.codes.shape == (0, 7, 64) and torch.equal(mx.product(flat, flat), torch.zeros(7, 7, device=DEV))
    assert torch.equal(mx.product(flat, flat, out=torch.ones(7, 7, device=DEV), accumulate=True), torch.ones(7, 7, device=DEV))
    assert mx.unpack(flat).shape == (7, 0)
    assert mx.pack(torch.empty(7, 0, device=DEV), transposed=True).shape == (0, 7)


def test_offsets_past_32_bits():
    mx = micro.Microscaled()
    # 9 GB of codes
    rows, cols = 2 ** 24, 1024
    codes = torch.zeros(8, rows, 64, dtype=torch.uint8, device=DEV)
    scales = torch.full((8, rows, 4), 127, dtype=torch.uint8, device=DEV)
    codes[-1, -1, -1] = 0x20  # 1 in the last value
    scales[-1, -1, -1] = 130
    big = micro.PackedMatrix(codes, scales, rows, cols)
    one = torch.zeros(1, cols, device=DEV)
    one[0, -1] = 3.0
    got = mx.linear(one, big, dtype=torch.float32)
    assert float(got[0, -1]) == 24.0 and float(got.abs().sum()) == 24.0
    last = mx.unpack(micro.PackedMatrix(codes[:, -5:].contiguous(), scales[:, -5:].contiguous(), 5, cols))
    assert float(last[-1, -1]) == 8.0 and float(last.sum()) == 8.0
    del codes, scales, big, got
    # an output of 2.4e9 values
    a = mx.pack(torch.ones(80_000, 32, device=DEV))
    b = mx.pack(torch.full((30_000, 32), 2.0, device=DEV))
    out = mx.product(a, b, dtype=torch.bfloat16)
    assert float(out.amin()) == 64.0 and float(out.amax()) == 64.0
    del out
    # 2.4e9 values packed both ways
    x = torch.zeros(70_000, 35_000, dtype=torch.bfloat16, device=DEV)
    x[-1, -1] = 2.0
    q, t = mx.pack_both(x)
    del x
    probe = torch.zeros(1, 35_000, device=DEV)
    probe[0, -1] = 1.0
    got = mx.linear(probe, q, dtype=torch.float32)
    assert float(got[0, -1]) == 2.0 and float(got.abs().sum()) == 2.0
    probe = torch.zeros(1, 70_000, device=DEV)
    probe[0, -1] = 1.0
    got = mx.linear(probe, t, dtype=torch.float32)
    assert float(got[0, -1]) == 2.0 and float(got.abs().sum()) == 2.0


def test_backward_products_are_the_derivative():
    """y = x w^T on values that are exact in 4 bits: the two products are the
    gradients of L = sum(y d), against the formula and central differences in 64
    bits (L is bilinear: exact up to rounding)."""
    gen = torch.Generator().manual_seed(3)
    level = lambda *s: ref.LEVELS[torch.randint(0, 8, s, generator=gen)] * (1 - 2 * torch.randint(0, 2, s, generator=gen))  # noqa: E731
    x, w, d = level(50, 70), level(33, 70), level(50, 33)
    for t in (x, w, d):  # every block along either side has scale 1
        t[::16], t[:, ::16] = 4.0, 4.0
    mx = micro.Microscaled()
    f = lambda t: t.float().to(DEV)  # noqa: E731
    dx = mx.product(mx.pack(f(d)), mx.pack(f(w), transposed=True)).cpu().double()
    dw = mx.product(mx.pack(f(d), transposed=True), mx.pack(f(x), transposed=True)).cpu().double()
    assert torch.equal(dx, d @ w) and torch.equal(dw, d.t() @ x)
    for t, grad in ((x, dx), (w, dw)):
        step = torch.randn(t.shape, generator=gen).double()
        loss = lambda s: float((((x + s * step) @ w.t() if t is x else x @ (w + s * step).t()) * d).sum())  # noqa: E731, B023
        slope = (loss(1e-3) - loss(-1e-3)) / 2e-3
        assert abs(slope - float((grad * step).sum())) <= 1e-9 * float((grad.abs() * step.abs()).sum())


def test_another_stream_and_a_captured_graph():
    gen = torch.Generator().manual_seed(9)
    x = torch.randn(70, 400, generator=gen).to(DEV)
    w = torch.randn(600, 400, generator=gen).to(DEV)
    mx = micro.Microscaled()
    want = mx.linear(x, mx.pack(w))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    other = micro.Microscaled(stream=stream)
    got = other.linear(x, other.pack(w))  # the current stream is not the handle's
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got, want)
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            q, t = other.pack_both(w)
            y = other.linear(x, q)
            z = other.product(t, t)
    for i in range(4):
        x.copy_(torch.randn(70, 400, generator=gen))
        w.mul_(1.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, mx.linear(x, mx.pack(w)))
        wt = mx.pack(w, transposed=True)
        assert torch.equal(z, mx.product(wt, wt))


def test_refusals():
    mx = micro.Microscaled()
    x = torch.ones(8, 64, device=DEV)
    q, other = mx.pack(x), mx.pack(torch.ones(8, 32, device=DEV))
    out = torch.full((8, 8), 7.0, device=DEV)
    for call, error in [(lambda: mx.pack(x.double()), TypeError), (lambda: mx.pack(x.cpu()), TypeError),
                        (lambda: mx.pack(x.t()), TypeError), (lambda: mx.pack(x[:, ::2]), TypeError),
                        (lambda: mx.product(q, other), micro.MicroError), (lambda: mx.product(q, x), TypeError),
                        (lambda: mx.product(q, q, dtype=torch.float64), TypeError),
                        (lambda: mx.product(q, q, out=out[:4]), ValueError),
                        (lambda: mx.product(q, q, dtype=torch.float16, out=out), TypeError),
                        (lambda: mx.product(q, q, accumulate=True), ValueError),
                        (lambda: mx.linear(x[:, :32], q), ValueError),
                        (lambda: mx.unpack(q, out=out), ValueError),
                        (lambda: mx.product(q, q, out=q.codes.view(torch.float32).view(8, 16)[:, :8]), (micro.MicroError, ValueError)),
                        (lambda: mx.pack(torch.nn.Parameter(x)), RuntimeError),
                        (lambda: mx.linear(x, q, out=torch.nn.Parameter(out)), RuntimeError)]:
        with pytest.raises(error):
            call()
    torch.cuda.synchronize()
    assert bool((out == 7).all())
    with torch.no_grad():
        assert torch.equal(mx.unpack(mx.pack(torch.nn.Parameter(x))), x)
    mx.close()
    with pytest.raises(RuntimeError, match="closed"):
        mx.pack(x)


@pytest.mark.parametrize("change,error", changes_in_place())
def test_matrices_whose_tensors_were_changed_in_place_are_refused(change, error):
    """On the native way and on the other, before anything is read."""
    mx = micro.Microscaled()
    x = torch.ones(40, 300, device=DEV)
    whole = mx.pack(x)
    out = torch.full((40, 40), 7.0, device=DEV)
    values = torch.full((40, 300), 7.0, device=DEV)
    for call in (lambda m: mx.product(m, whole), lambda m: mx.product(whole, m), lambda m: mx.linear(x, m), lambda m: mx.unpack(m),
                 lambda m: mx.product(m, whole, out=out), lambda m: mx.product(whole, m, out=out, accumulate=True),
                 lambda m: mx.linear(x, m, out=out), lambda m: mx.unpack(m, out=values)):
        m = mx.pack(x)
        change(m)
        with pytest.raises(error):
            call(m)
    for part in ("codes", "scales"):  # memory of the host
        m = mx.pack(x)
        getattr(m, part).data = getattr(m, part).cpu()
        for call in (lambda: mx.product(m, whole), lambda: mx.unpack(m), lambda: mx.linear(x, m, out=out)):
            with pytest.raises(TypeError):
                call()
    torch.cuda.synchronize()
    assert bool((out == 7).all()) and bool((values == 7).all())
    # other memory of the same shape is read from then on
    m = mx.pack(x)
    m.codes.data = mx.pack(x * 1.5).codes.clone()
    assert torch.equal(mx.unpack(m), x * 1.5) and torch.equal(mx.unpack(m, out=values), x * 1.5)
    assert torch.equal(mx.product(m, whole), torch.full((40, 40), 450.0, device=DEV))
