"""What the norm's layers return is written once, by the kernel: no copy is made of it, at widths that are no whole 16 bytes either."""
import pytest
import torch

from paper_2607_24953_b200 import autograd

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def peak(f):
    f()
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    kept = f()
    torch.cuda.synchronize()
    return torch.cuda.max_memory_allocated() - before, kept


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1999, 2731), (2000, 2736), (513, 4097)])
def test_the_norms_outputs_are_not_copied(rows, cols, dtype):
    x, r, g = randn(1, rows, cols).to(dtype), randn(2, rows, cols).to(dtype), 1 + 0.2 * randn(3, cols)
    for residual in (None, r):
        most, out = peak(lambda: autograd.rms_norm(x, g, residual))
        outs = [out] if residual is None else list(out)
        assert all(t.is_contiguous() for t in outs)
        # the outputs and 1 / root of every row, each in whole blocks of the allocator's (2 MB at most)
        assert most <= sum(t.numel() * t.element_size() for t in outs) + (len(outs) + 1) * (2 << 20)


@pytest.mark.parametrize("rows,cols", [(1999, 2731), (4001, 1027)])
def test_the_stream_is_not_copied(rows, cols):
    x, r, g, w = randn(1, rows, cols).to(BF16), randn(2, rows, cols), 1 + 0.2 * randn(3, cols), randn(4, 64, cols) * 0.05
    most, (y, h) = peak(lambda: autograd.rms_norm_fp8_linear(x, g, w, r))
    assert y.is_contiguous() and h.is_contiguous()
    codes = rows * (cols + 16) + 64 * (cols + 16)
    assert most <= h.numel() * 4 + codes + 2 * y.numel() * 2 + 8 * (2 << 20)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_nothing_is_kept_for_a_backward_pass_where_gradients_are_off(dtype):
    rows, cols, n = 4096, 2048, 512
    x, g, w = randn(1, rows, cols).to(dtype).requires_grad_(), (1 + 0.2 * randn(3, cols)).requires_grad_(), (randn(4, n, cols) * 0.05).requires_grad_()
    for f in (lambda: autograd.fp8_linear(x, w), lambda: autograd.rms_norm_fp8_linear(x, g, w)):
        want = f().detach()
        with torch.no_grad():
            most, y = peak(f)
        assert torch.equal(y, want)
        # codes and scales of x and of the weight, the output, 1 / root of every row
        assert most <= (rows + n) * cols + rows * (cols // 128) * 4 + y.numel() * 2 + 6 * (2 << 20)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", [64, 70, 75, 9001])
def test_outputs_may_be_changed_in_place(cols, dtype):
    x, r, g, w = randn(1, 30, cols).to(dtype).requires_grad_(), randn(2, 30, cols).to(dtype).requires_grad_(), (1 + 0.2 * randn(3, cols)).requires_grad_(), (randn(4, 20, cols) * 0.05).requires_grad_()
    for f in (lambda: autograd.rms_norm(x, g), lambda: autograd.rms_norm(x, g, r)[0], lambda: autograd.fp8_linear(x, w), lambda: autograd.rms_norm_fp8_linear(x, g, w), lambda: autograd.rms_norm_fp8_linear(x, g, w, r)[0]):
        x.grad = None
        y = f()
        y.mul_(2)
        y.sum().backward()
        got, x.grad = x.grad, None
        (f() * 2).sum().backward()
        assert torch.equal(got, x.grad)
