"""The norm, the 8-bit linear layer and the clipping as they are used together: one training step, eager, on another stream, in a captured graph."""
import pytest
import torch

from paper_2607_24953_b200 import autograd, binding as b

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def params(n, k, seed=0):
    return (1 + 0.2 * randn(seed, k)).requires_grad_(), (randn(seed + 1, n, k) * 0.05).requires_grad_()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(6, 40), (2, 3, 500), (0, 64), (700,)])
def test_the_norms_gradients(shape, dtype):
    x, r = randn(1, *shape).to(dtype).requires_grad_(), randn(2, *shape).to(dtype).requires_grad_()
    w = (1 + 0.2 * randn(3, shape[-1])).requires_grad_()
    dy, dh = randn(4, *shape).to(dtype), randn(5, *shape).to(dtype)
    if len(shape) == 1:
        with pytest.raises(ValueError):
            autograd.rms_norm(x, w[:-1], r)
    y, h = autograd.rms_norm(x, w, r)
    assert y.shape == h.shape == x.shape and y.dtype == h.dtype == dtype
    torch.autograd.backward([y, h], [dy, dh])
    X, R, W = (t.detach().double().requires_grad_() for t in (x, r, w))
    H = X + R
    H = H + (h.detach().double() - H.detach())           # as it was rounded
    Y = H * torch.rsqrt(H.square().mean(-1, keepdim=True) + 1e-6) * W
    torch.autograd.backward([Y, H], [dy.double(), dh.double()])
    half = torch.finfo(dtype).eps / 2
    for got, want in ((y, Y), (x.grad, X.grad), (r.grad, R.grad)):
        assert got.dtype == dtype
        # one rounding to the type, and FP32's along a row
        assert ((got.double() - want).abs() <= want.abs() * half + (want.abs() + dy.abs().max().double() * 8 if dy.numel() else 0) * 600 * 2.0 ** -24).all()
    assert (w.grad.double() - W.grad).abs().max() <= 1e-5 * max(1.0, float(W.grad.abs().max())) if W.grad.numel() else True


def test_the_layer_is_its_calls():
    x, (_, w) = randn(1, 300, 520).to(BF16).requires_grad_(), params(260, 520)
    dy = randn(2, 300, 260).to(BF16)
    y = autograd.fp8_linear(x, w)
    y.backward(dy)
    X, W, D = b.fp4q_fp8_quantize(x.detach()), b.fp4q_fp8_quantize(w.detach(), square=True), b.fp4q_fp8_quantize(dy)
    assert torch.equal(y, b.fp4q_fp8_gemm_fwd(X, W))
    assert torch.equal(x.grad, b.fp4q_fp8_gemm_dgrad(D, W)) and torch.equal(w.grad, b.fp4q_fp8_gemm_wgrad(D, X))
    assert x.grad.dtype == BF16 and w.grad.dtype == F32
    # against the layer without 8 bits: every element of an operand is off by half a step at most, 2^-4 of itself (or 2^-10 of 448 parts of its block's largest), in random directions
    full = x.detach().double() @ w.detach().double().T
    assert float((y.double() - full).norm() / full.norm()) < 2 * 2.0 ** -4
    x3 = x.detach().view(3, 100, 520)
    assert torch.equal(autograd.fp8_linear(x3, w).view(300, 260), y)
    assert torch.equal(autograd.fp8_linear(x.detach().T.contiguous().T, w), y)      # rows that are not contiguous


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows", [1, 77, 0])
def test_the_norm_in_front_of_the_layer_is_its_calls(rows, residual):
    x, r = randn(1, rows, 328).to(BF16).requires_grad_(), randn(2, rows, 328).requires_grad_() if residual else None
    g, w = params(200, 328)
    out = autograd.rms_norm_fp8_linear(x, g, w, r)
    y, h = out if residual else (out, None)
    n = b.fp4q_rms_norm(x.detach(), g.detach(), None if r is None else r.detach(), q=b.Q_FP8, rstd=True)
    W = b.fp4q_fp8_quantize(w.detach(), square=True)
    assert torch.equal(y, b.fp4q_fp8_gemm_fwd(b.Fp8Tensor(rows, 328, n.q, n.scale), W))
    assert not residual or torch.equal(h, n.h)
    dy, dh = randn(3, rows, 200).to(BF16), randn(4, rows, 328) if residual else None
    torch.autograd.backward([y, h] if residual else [y], [dy, dh] if residual else [dy])
    D, X = b.fp4q_fp8_quantize(dy), b.fp4q_fp8_quantize(n.y, want=False)
    dx, dg = b.fp4q_rms_norm_bwd(b.fp4q_fp8_gemm_dgrad(D, W), n.h if residual else x.detach(), n.rstd, g.detach(), dh=dh)
    assert torch.equal(x.grad, dx.to(BF16)) and torch.equal(g.grad, dg) and torch.equal(w.grad, b.fp4q_fp8_gemm_wgrad(D, X))
    assert not residual or torch.equal(r.grad, dx)


def test_only_the_gradients_that_are_wanted():
    x, (g, w) = randn(1, 50, 128).to(BF16), params(64, 128)
    for need in range(8):
        X, G, W = (t.detach().clone().requires_grad_(bool(need >> i & 1)) for i, t in enumerate((x, g, w)))
        y = autograd.rms_norm_fp8_linear(X, G, W)
        assert y.requires_grad == (need > 0)
        if need:
            y.backward(torch.ones_like(y))
        for i, t in enumerate((X, G, W)):
            assert (t.grad is not None) == bool(need >> i & 1)


def test_outputs_that_nobody_uses_get_no_gradient():
    x, r, (g, w) = randn(1, 30, 64).to(BF16).requires_grad_(), randn(2, 30, 64).to(BF16).requires_grad_(), params(48, 64)
    for f in (lambda: autograd.rms_norm(x, g, r), lambda: autograd.rms_norm_fp8_linear(x, g, w, r)):
        both = []
        for use in (0, 1):
            x.grad = r.grad = None
            f()[use].sum().backward()
            both.append((x.grad, r.grad))
        assert torch.equal(both[0][0], both[0][1])
        assert (both[1][0] == 1).all() and (both[1][1] == 1).all()      # the stream's own gradient alone


class Block:
    """Two projections behind norms on one residual stream, a step's gradients clipped and turned into updates."""

    def __init__(self, rows, k, n):
        self.x, self.r = randn(1, rows, k).to(BF16), randn(2, rows, k).to(BF16)
        self.g1, self.w1 = params(n, k, 10)
        self.g2, self.w2 = params(k, n, 20)
        self.ps = [self.g1, self.w1, self.g2, self.w2]
        self.target, self.ws = randn(3, rows, k), b.alloc_workspace("cuda")

    def step(self):
        for p in self.ps:
            p.grad = None
        a, h = autograd.rms_norm_fp8_linear(self.x, self.g1, self.w1, self.r, ws=self.ws)
        y = autograd.rms_norm_fp8_linear(torch.nn.functional.silu(a), self.g2, self.w2, ws=self.ws)
        z, _ = autograd.rms_norm(y, None, h)
        ((z.float() - self.target) ** 2).mean().backward()
        norm = autograd.clip_grad_norm_(self.ps, 0.01)
        return [z.detach(), norm] + [p.grad for p in self.ps] + [b.fp4q_newton_schulz(p.grad, ws=self.ws) for p in (self.w1, self.w2)]


@pytest.mark.parametrize("rows,k,n", [(40, 256, 512), (333, 500, 390)])
def test_a_step_eager_on_another_stream_and_captured(rows, k, n):
    block = Block(rows, k, n)
    want = [t.clone() for t in block.step()]
    assert all(t.isfinite().all() for t in want) and float(want[1]) > 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [t.clone() for t in block.step()]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        for p in block.ps:
            p.grad = None
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block.step()
    for scale in (1.0, 2.0):
        with torch.no_grad():
            block.target.mul_(scale)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        if scale == 1.0:
            assert all(torch.equal(p, q) for p, q in zip(got, want))
        else:
            assert torch.equal(got[0], want[0]) and not torch.equal(got[1], want[1])
    assert b.fp4q_workspace_status(block.ws) == 0


def test_calls_in_a_stream_that_is_given():
    x, (g, w) = randn(1, 200, 384).to(BF16), params(256, 384)
    g, w = g.detach(), w.detach()
    W = b.fp4q_fp8_quantize(w, square=True)

    def run(stream):
        n = b.fp4q_rms_norm(x, g, x, q=b.Q_FP8, rstd=True, stream=stream)
        y = b.fp4q_fp8_gemm_fwd(b.Fp8Tensor(200, 384, n.q, n.scale), W, stream=stream)
        t = b.fp4q_fp8_quantize(y, stream=stream)
        dx, dw = b.fp4q_rms_norm_bwd(b.fp4q_fp8_gemm_dgrad(t, W, stream=stream), n.h, n.rstd, g, stream=stream)
        gw = b.fp4q_fp8_gemm_wgrad(t, b.fp4q_fp8_quantize(n.y, stream=stream), stream=stream)
        norm = b.fp4q_clip_grad_norm([dx, dw, gw], 1.0, stream=stream)
        return [y, dx, dw, gw, norm]
    want = run(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got = run(side)
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_chains_without_synchronisation_match_synchronised_ones():
    xs = [randn(i, 130, 256).to(BF16) for i in range(4)]
    (g, w), ws = params(130, 256), b.alloc_workspace("cuda")
    g, w = g.detach(), w.detach()
    W = b.fp4q_fp8_quantize(w, square=True)
    x, out = torch.empty_like(xs[0]), b.alloc_norm(xs[0], xs[0], q=b.Q_FP8, rstd=True)
    q, y = b.alloc_fp8tensor(130, 130, "cuda"), torch.empty(130, 136, dtype=BF16, device="cuda")[:, :130]

    def run(after):
        kept = []
        for i in range(20):
            for call in (lambda: x.copy_(xs[i % 4]), lambda: b.fp4q_rms_norm(x, g, xs[0], out=out), lambda: x.zero_(),
                         lambda: b.fp4q_fp8_gemm_fwd(b.Fp8Tensor(130, 256, out.q, out.scale), W, out=y, ws=ws), lambda: out.q.zero_(),
                         lambda: b.fp4q_fp8_quantize(y, out=q), lambda: y.zero_(), lambda: kept.append(b.fp4q_fp8_gemm_dgrad(q, W, ws=ws)),
                         lambda: kept.append(b.fp4q_global_norm([kept[-1]])), lambda: kept.append(b.fp4q_rms_norm_bwd(kept[-2], out.h, out.rstd, g)[1])):
                call()
                after()
        return kept
    a = run(torch.cuda.synchronize)
    c = run(lambda: None)
    assert all(torch.equal(p, q) for p, q in zip(a, c))
