"""The layer of ragged groups: gradients in the precision of what they belong to, inputs and gradients in any strides."""
import math

import pytest
import torch

from paper_2607_24953_b200 import autograd, binding as b

pytestmark = pytest.mark.gpu


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def test_an_fp32_input_gets_an_fp32_gradient():
    # An accumulator's instruction is off by less than 2^-22 of the sum of the absolute products, and there are n / 16 in one; the sum is rounded once.
    T, n, k, spans = 300, 72, 100, [(0, 50), (50, 180), (180, 300)]
    offs = torch.tensor([0, 50, 180, 300], device="cuda")
    x, w = randn(1, T, k).requires_grad_(), randn(2, 3, n, k) * 0.1
    dy = randn(3, T, n).to(torch.bfloat16)
    autograd.ragged_linear(x, w, offs).backward(dy)
    for g, (i, j) in enumerate(spans):
        m = w[g].bfloat16().double()
        want, s = dy[i:j].double() @ m, dy[i:j].double().abs() @ m.abs()
        assert ((x.grad[i:j].double() - want).abs() <= s * (math.ceil(n / 16) * 2 ** -22 + 2 ** -24)).all()


def test_a_single_column_in_any_strides_and_an_expanded_gradient():
    offs, spans = torch.tensor([0, 30, 64], device="cuda"), [(0, 30), (30, 64)]
    x = randn(1, 64, 64).to(torch.bfloat16)[:, ::8][:, :1].detach().requires_grad_()
    w = randn(2, 2, 1, 8).to(torch.bfloat16)[:, :, :1].detach().requires_grad_()          # one column in, one column out
    y = autograd.ragged_linear(x, w, offs)
    y.sum().backward()                                       # ones in strides of zero
    for g, (i, j) in enumerate(spans):
        assert torch.equal(y[i:j], x.detach()[i:j] * w.detach()[g])                        # a product is rounded once
        assert torch.equal(x.grad[i:j], w.detach()[g].expand(j - i, 1))
        want, s = x.detach()[i:j].double().sum(), x.detach()[i:j].double().abs().sum()
        assert abs(w.grad[g].double() - want) <= abs(want) * 2 ** -8 + s * 3 * 2 ** -22
    dy = randn(3, 64, 24).to(torch.bfloat16)[:, ::8][:, :1]
    y = autograd.ragged_linear(x, w, offs)
    x.grad = None
    y.backward(dy)
    assert torch.equal(x.grad[:30], dy[:30] * w.detach()[0])
