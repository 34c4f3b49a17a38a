"""What types the norm's and the 8-bit layers take, without a device."""
import pytest
import torch

from paper_2607_24953_b200 import autograd


def test_other_types_become_fp32_and_numbers_that_are_not_floating_point_are_refused():
    for dtype in (torch.float16, torch.float64, torch.float8_e4m3fn):
        t = torch.tensor([[1.0, 0.125, 3.5]]).to(dtype)
        assert autograd._rows(t).dtype == torch.float32 and torch.equal(autograd._rows(t), t.float())
    # 1 + 2^-10 is an FP16 number that BF16 does not have
    assert float(autograd._rows(torch.full((2, 2), 1 + 2.0 ** -10, dtype=torch.float16))[0, 0]) == 1 + 2.0 ** -10
    assert float(autograd._weight(torch.full((2,), 1 + 2.0 ** -10, dtype=torch.float16))[0]) == 1 + 2.0 ** -10
    for dtype in (torch.int32, torch.bool, torch.complex64):
        t = torch.ones(2, 2).to(dtype)
        for call in (lambda: autograd._rows(t), lambda: autograd._weight(t[0]), lambda: autograd.rms_norm(t), lambda: autograd.fp8_linear(torch.ones(2, 2), t)):
            with pytest.raises(ValueError):
                call()
