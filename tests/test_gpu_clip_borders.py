"""The clipping of gradients at the borders of what it takes."""
import pytest
import torch

from paper_2607_24953_b200 import autograd, binding as b

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("max_norm", [0.0, 1.0, float("inf")])
def test_zeros_stay_zeros_without_an_eps(max_norm, dtype):
    g = [torch.zeros(50, dtype=dtype, device="cuda"), torch.zeros(9000, dtype=dtype, device="cuda")]
    outs = [torch.ones(t.shape, device="cuda") for t in g]
    assert float(b.fp4q_clip_grad_norm(g, max_norm, outs=outs, eps=0.0)) == 0 and not any(t.any() for t in outs)
    assert float(b.fp4q_clip_grad_norm(g, max_norm, eps=0.0)) == 0 and not any(t.any() for t in g)
    b.fp4q_clip_by_norm(g, torch.zeros((), device="cuda"), max_norm, eps=0.0)
    assert not any(t.any() for t in g)


def test_the_norm_of_no_gradients_is_on_the_parameters_device():
    p = torch.nn.Parameter(torch.ones(5, device="cuda"))
    for norm in (autograd.clip_grad_norm_([p], 1.0), autograd.clip_grad_norm_(p, 1.0), autograd.clip_grad_norm_(iter([p, p]), 1.0)):
        assert norm.device == p.device and norm.dtype == F32 and norm.shape == () and float(norm) == 0
    assert autograd.clip_grad_norm_([], 1.0) == 0
