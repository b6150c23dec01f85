"""A gradient set keeps the memory that it was made for."""
import pytest
import torch

import paper_2310_00967_amd as micro

pytestmark = pytest.mark.gpu

DEV = "cuda"


def test_a_tensor_that_is_given_other_memory():
    """`data` swapped behind the set's back: what the set reads and writes stays
    allocated, and no other tensor gets it."""
    a = torch.full((3_000_000,), 2.0, device=DEV)
    b = torch.full((500,), 3.0, device=DEV, dtype=torch.bfloat16)
    grads = micro.GradientSet([a, b])
    want = float(grads.norm())
    at = {a.data_ptr(), b.data_ptr()}
    a.data = torch.zeros(3_000_000, device=DEV)
    b.data = torch.zeros(500, device=DEV, dtype=torch.bfloat16)
    others = [torch.full((n,), 5.0, device=DEV, dtype=t) for n, t in ((3_000_000, a.dtype), (500, b.dtype)) for _ in range(20)]
    assert not at & {t.data_ptr() for t in others}
    assert float(grads.norm()) == want
    grads.clip_(1.0)
    torch.cuda.synchronize()
    assert all(bool((t == 5.0).all()) for t in others) and bool((a == 0).all()) and bool((b == 0).all())
