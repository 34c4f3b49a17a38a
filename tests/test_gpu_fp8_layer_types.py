"""The norm and the 8-bit layer in one call and in two, and tensors of types other than BF16 and FP32."""
import pytest
import torch

from paper_2607_24953_b200 import autograd

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("stream", [None, BF16, F32])
@pytest.mark.parametrize("rows,k,n", [(1, 40, 24), (77, 328, 200), (300, 515, 130), (9, 9000, 32)])
def test_on_fp32_one_call_is_the_two_calls(rows, k, n, stream):
    x, g, w = randn(1, rows, k).requires_grad_(), (1 + 0.2 * randn(2, k)).requires_grad_(), (randn(3, n, k) * 0.05).requires_grad_()
    r = None if stream is None else randn(4, rows, k).to(stream).requires_grad_()
    dy, dh = randn(5, rows, n).to(BF16), None if r is None else randn(6, rows, k).to(stream)
    leaves = [t for t in (x, g, w, r) if t is not None]
    both = []
    for fused in (True, False):
        if fused:
            out = autograd.rms_norm_fp8_linear(x, g, w, r)
            y, h = (out, None) if r is None else out
        else:
            out = autograd.rms_norm(x, g, r)
            a, h = (out, None) if r is None else out
            y = autograd.fp8_linear(a, w)
        outs, grads = ([y], [dy]) if r is None else ([y, h], [dy, dh])
        both.append(outs + list(torch.autograd.grad(outs, leaves, grads)))
    for p, q in zip(*both):
        assert p.dtype == q.dtype and torch.equal(p, q)


def run(f, leaves, grads):
    leaves = [t.detach().requires_grad_() for t in leaves]
    out = f(*leaves)
    outs = list(out) if isinstance(out, tuple) else [out]
    return outs, torch.autograd.grad(outs, leaves, grads[:len(outs)])


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64])
def test_other_types_are_computed_in_fp32(dtype):
    x, r, g, w = randn(1, 50, 76).to(dtype), randn(2, 50, 76).to(dtype), (1 + 0.2 * randn(3, 76)).to(dtype), (randn(4, 40, 76) * 0.05).to(dtype)
    dy, dz, dh = randn(5, 50, 76).to(dtype), randn(6, 50, 40).to(BF16), randn(7, 50, 76).to(dtype)
    cases = [(autograd.rms_norm, [x, g], [dy]), (autograd.rms_norm, [x, g, r], [dy, dh]), (autograd.fp8_linear, [x, w], [dz]), (autograd.rms_norm_fp8_linear, [x, g, w], [dz]),
             (autograd.rms_norm_fp8_linear, [x, g, w, r], [dz, dh])]
    for f, leaves, grads in cases:
        outs, got = run(f, leaves, grads)
        wide, want = run(f, [t.float() for t in leaves], [t if t.dtype == BF16 else t.float() for t in grads])
        for p, q in zip(outs, wide):
            assert p.dtype == (BF16 if q.dtype == BF16 else dtype) and torch.equal(p, q.to(p.dtype))
        for p, q in zip(got, want):
            assert p.dtype == dtype and torch.equal(p, q.to(dtype))
