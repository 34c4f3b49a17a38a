"""What the ragged layer and its binding make of their arguments, without a device."""
import pytest
import torch

from paper_2607_24953_b200 import autograd, binding as b


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_operands_are_brought_into_rows_that_the_products_take(dtype):
    big = torch.arange(6 * 64).reshape(6, 64).to(dtype)
    views = [big, big[:, 8:40], big[:, 3:], big[:, ::8][:, :1], big[:, :1], big[1:2, ::2], big.T, big.T[:, :1], big[:, :0], big[:0], big[:1].expand(5, 64),
             big[:, :1].expand(6, 9)]
    for t in views:
        r = autograd._rows16(t)
        assert r.dtype == torch.bfloat16 and torch.equal(r, t.to(torch.bfloat16))
        if r.numel():
            assert r.stride(1) == 1 and r.stride(0) % 8 == 0 and r.stride(0) >= r.shape[1] and r.data_ptr() % 16 == 0
    t = torch.zeros(6, 64, dtype=torch.bfloat16)
    assert autograd._rows16(t) is t                          # nothing is copied that need not be
