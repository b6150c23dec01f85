"""Arguments of the token table that lie in one buffer: columns that share no
value are separate arguments, rows that share one are refused."""
import pytest
import torch

import paper_2310_00967_amd as micro
from paper_2310_00967_amd import _lib

pytestmark = pytest.mark.gpu

DEV = "cuda"


def inputs(dtype):
    gen = torch.Generator().manual_seed(1)
    hidden = torch.randn(20, 64, generator=gen).to(dtype)
    weight = torch.randn(30, 64, generator=gen).mul_(0.1).to(dtype)
    return hidden.to(DEV), weight.to(DEV), torch.randint(0, 30, (20,), generator=gen).to(DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_columns_of_one_buffer_are_apart(dtype):
    hidden, weight, ids = inputs(dtype)
    table = micro.TokenTable(30, 64, 20, dtype=dtype)
    packed = torch.zeros(30, 4 * 64, dtype=dtype, device=DEV)  # weight, dweight, hidden, dhidden
    w, dw, h, dh = (packed[:n, a:a + 64] for n, a in ((30, 0), (30, 64), (20, 128), (20, 192)))
    w.copy_(weight), h.copy_(hidden)
    got = table.loss_grad(h, w, ids, dhidden=dh, dweight=dw)
    want = table.loss_grad(hidden, weight, ids)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert torch.equal(w, weight) and torch.equal(h, hidden)
    table.lookup(w, ids, out=dh)
    assert torch.equal(dh, weight[ids])
    table.lookup_grad(h, ids, dw)
    assert torch.equal(dw, table.lookup_grad(hidden, ids, torch.empty_like(weight)))
    assert torch.equal(w, weight) and torch.equal(h, hidden)


def test_rows_that_share_a_value_are_refused():
    hidden, weight, ids = inputs(torch.float32)
    table = micro.TokenTable(30, 64, 20)
    packed = torch.zeros(41, 128, device=DEV)
    flat = packed.view(-1)
    h = packed[:20, :64]
    for out in (packed[:20, 63:127], packed[19:39, :64], flat[65:].as_strided((20, 64), (128, 1)),
                flat.as_strided((20, 64), (130, 1), 64)):
        with pytest.raises(_lib.MicroError) as e:
            table.loss_grad(h, weight, ids, dhidden=out)
        assert e.value.status == _lib.MICRO_EINVAL and "memory" in str(e.value)
    torch.cuda.synchronize()
    assert bool((packed == 0).all())
    table.loss_grad(h, weight, ids, dhidden=packed[20:40, :64])  # behind its last row
