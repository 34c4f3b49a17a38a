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
