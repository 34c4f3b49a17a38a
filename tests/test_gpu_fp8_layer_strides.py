"""The norm's and the 8-bit layers on tensors whose rows share memory, as sums and expanded inputs leave them: the results are those of contiguous copies, bit for bit."""
import pytest
import torch

from paper_2607_24953_b200 import autograd

BF16, F32 = torch.bfloat16, torch.float32
K, N = 96, 40


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def test_rows_are_taken_where_they_are_or_copied():
    base = torch.arange(40.0)
    for t in (base.view(5, 8), base.view(5, 8)[:, :6], base.view(5, 8)[:1], base.view(5, 8)[:, :1], base.view(8, 5)[2:, 1:4].to(BF16), base[:0].view(0, 8), base[:0].view(8, 0)):
        assert autograd._rows(t) is t
    for t in (base[:8].expand(5, 8), base[:1].expand(5, 1), base[:1].expand(5, 8), base.as_strided((5, 8), (1, 1)), base.as_strided((5, 8), (7, 1)), base.view(8, 5).T):
        rows = autograd._rows(t)
        assert rows.is_contiguous() and torch.equal(rows, t)


def windows(t, rows, cols):
    """Rows that begin one element behind each other."""
    return t.as_strided((rows, cols), (1, 1))


def layers(dtype):
    g, w = (1 + 0.2 * randn(10, K)).requires_grad_(), (randn(11, N, K) * 0.05).requires_grad_()
    return {"norm": (lambda x, r: autograd.rms_norm(x, g), [g], K), "norm and stream": (lambda x, r: autograd.rms_norm(x, g, r), [g], K),
            "linear": (lambda x, r: autograd.fp8_linear(x, w), [w], N), "norm and linear": (lambda x, r: autograd.rms_norm_fp8_linear(x, g, w, r), [g, w], N)}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("name", ["norm", "norm and stream", "linear", "norm and linear"])
@pytest.mark.parametrize("rows", [1, 33, 300])
def test_gradients_whose_rows_share_memory(name, dtype, rows):
    f, leaves, n = layers(dtype)[name]
    x, r = randn(1, rows, K).to(dtype).requires_grad_(), randn(2, rows, K).to(dtype).requires_grad_()
    out = f(x, r)
    outs = list(out) if isinstance(out, tuple) else [out]
    long = [randn(3 + i, rows + o.shape[1]).to(o.dtype) for i, o in enumerate(outs)]
    for grads in ([t[:o.shape[1]].expand_as(o) for t, o in zip(long, outs)], [t[:1].expand_as(o) for t, o in zip(long, outs)], [windows(t, *o.shape) for t, o in zip(long, outs)]):
        got = torch.autograd.grad(f_outs(f, x, r), [x, r] + leaves, grads, allow_unused=True)
        want = torch.autograd.grad(f_outs(f, x, r), [x, r] + leaves, [t.contiguous() for t in grads], allow_unused=True)
        for p, q in zip(got, want):
            assert (p is None) == (q is None) and (p is None or torch.equal(p, q))


def f_outs(f, x, r):
    out = f(x, r)
    return list(out) if isinstance(out, tuple) else [out]


@pytest.mark.gpu
def test_sums_over_tokens():
    x, r = randn(1, 50, K).to(BF16).requires_grad_(), randn(2, 50, K).to(BF16).requires_grad_()
    for name, (f, leaves, n) in layers(BF16).items():
        for i in range(len(f_outs(f, x, r))):
            f_outs(f, x, r)[i].sum(0).backward(torch.ones_like(f_outs(f, x, r)[i][0]))
    w = (randn(3, 1, K) * 0.05).requires_grad_()
    autograd.fp8_linear(x, w).sum().backward()        # one column: every stride is 0
    y = autograd.fp8_linear(x, w)
    assert torch.equal(w.grad, torch.autograd.grad(y, w, torch.ones(50, 1, dtype=BF16, device="cuda"))[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("name", ["norm", "norm and stream", "linear", "norm and linear"])
def test_inputs_whose_rows_share_memory(name, dtype):
    f, leaves, n = layers(dtype)[name]
    a, c = randn(1, 200).to(dtype), randn(2, 200).to(dtype)
    for x, r in ((a[:K].expand(70, K), c[:K].expand(70, K)), (windows(a, 70, K), windows(c, 70, K)), (a[:1].expand(70, K), c[:1].expand(70, K))):
        for p, q in zip(f_outs(f, x, r), f_outs(f, x.contiguous(), r.contiguous())):
            assert torch.equal(p, q)


@pytest.mark.gpu
def test_weights_whose_rows_share_memory():
    x, a = randn(1, 30, K).to(BF16), randn(2, 200) * 0.05
    for w in (a[:K].expand(N, K), windows(a, N, K)):
        assert torch.equal(autograd.fp8_linear(x, w), autograd.fp8_linear(x, w.contiguous()))
    g = torch.ones(1, device="cuda").expand(K)
    assert torch.equal(autograd.rms_norm(x, g), autograd.rms_norm(x, g.contiguous()))
