"""What the 8-bit tensors' calls, the norm and the clipping refuse, without a device: the C entry points check their arguments before anything is enqueued, the binding its tensors."""
import ctypes

import pytest
import torch

from paper_2607_24953_b200 import autograd, binding as b

P = 0x100000


def tensor(rows=100, cols=200, square=0, **kw):
    f = dict(rows=rows, cols=cols, q=P, ld_q=208, scale=P, ld_s=2, q_t=P, ld_t=112, scale_t=P, ld_st=1, square=square)
    f.update(kw)
    return b._CFp8Tensor(*[f[n] for n, _ in b._CFp8Tensor._fields_])


def quantize(t, x=P, dt=0, rows=100, cols=200, ld=200):
    return b.lib().fp4q_fp8_quantize(x, dt, rows, cols, ld, ctypes.byref(t) if t else None, None)


def test_quantizer():
    t = tensor()
    assert quantize(None) == 1 and quantize(t, x=None) == 1 and quantize(tensor(q=None, q_t=None)) == 1
    assert quantize(t, rows=-1) == 2 and quantize(t, rows=99) == 2 and quantize(t, ld=199) == 2
    assert quantize(t, dt=2) == 4 and quantize(t, dt=0x100) == 4 and quantize(tensor(square=2)) == 4
    assert quantize(tensor(ld_q=192)) == 2 and quantize(tensor(ld_s=1)) == 2 and quantize(tensor(ld_t=96)) == 2 and quantize(tensor(ld_st=0)) == 2
    assert quantize(tensor(scale=None)) == 1 and quantize(tensor(scale_t=None)) == 1 and quantize(tensor(square=1, scale=None, q=None)) == 1
    assert quantize(t, x=P + 1) == 3 and quantize(t, x=P + 2, dt=1) == 3
    assert quantize(tensor(q=P + 8)) == 3 and quantize(tensor(q_t=P + 8)) == 3 and quantize(tensor(ld_q=200)) == 3 and quantize(tensor(ld_t=100)) == 3 and quantize(tensor(scale=P + 2)) == 3
    assert quantize(tensor(rows=0, q=None), x=None, rows=0) == 0


def product(which, x, y, c=P, ld=256, dt=1, acc=0, ws=P, wsb=256):
    f = [b.lib().fp4q_fp8_gemm_fwd, b.lib().fp4q_fp8_gemm_dgrad, b.lib().fp4q_fp8_gemm_wgrad][which]
    args = [ctypes.byref(x) if x else None, ctypes.byref(y) if y else None, c, ld, dt] + ([acc] if which == 2 else []) + [ws, wsb, None]
    return f(*args)


def test_products():
    X, W, dY = tensor(100, 200), tensor(160, 200, square=1, ld_t=160), tensor(100, 160, ld_q=160)
    pairs = [(X, W), (dY, W), (dY, X)]
    for which, (x, y) in enumerate(pairs):
        assert product(which, None, y) == 1 and product(which, x, None) == 1 and product(which, x, y, c=None) == 1
        assert product(which, x, y, ld=100) == 2 and product(which, x, y, dt=2) == 4 and product(which, x, y, dt=0x200) == 4
        assert product(which, x, y, c=P + 8) == 3 and product(which, x, y, ld=255) == 3
        assert product(which, x, y, ws=None) == 5 and product(which, x, y, wsb=8) == 5 and product(which, x, y, ws=P + 8) == 3
        assert product(which, tensor(-1, 200), y) == 2 and product(which, tensor(77, 77, ld_t=80), y) == 2
    assert product(0, tensor(100, 200, square=1), W) == 4 and product(0, X, tensor(160, 200)) == 4 and product(2, dY, tensor(100, 200, square=1)) == 4
    assert product(0, tensor(100, 200, q=None), W) == 1 and product(1, dY, tensor(160, 200, square=1, q_t=None)) == 1 and product(2, tensor(100, 160, scale_t=None), X) == 1
    assert product(0, tensor(100, 200, q=P + 1), W) == 3 and product(0, tensor(100, 200, ld_q=200), W) == 3 and product(0, tensor(100, 200, ld_q=192), W) == 2 and product(0, tensor(100, 200, ld_s=1), W) == 2
    assert product(2, dY, X, dt=0, acc=1) == 4
    assert product(0, tensor(0, 200), W, c=None, ws=None) == 0
    assert product(0, tensor(1 << 31, 200), W) == 4


def norm(rows=10, cols=300, **kw):
    f = dict(x=P, ld_x=300, x_type=0, residual=P, ld_residual=300, h=P, ld_h=300, h_type=1, weight=P, weight_type=1, eps=1e-6, y=P, ld_y=300, y_type=0, q=P, ld_q=320, scale=P, ld_s=10,
             q_format=1, rstd=P)
    f.update(kw)
    return b.lib().fp4q_rms_norm(ctypes.byref(b._CNorm(*[f[n] for n, _ in b._CNorm._fields_])), rows, cols, None)


def test_norm():
    assert b.lib().fp4q_rms_norm(None, 1, 1, None) == 1
    assert norm(rows=-1) == 2 and norm(cols=-1) == 2 and norm(cols=65537) == 4
    for k in ("x_type", "h_type", "weight_type", "y_type"):
        assert norm(**{k: 2}) == 4
    assert norm(q_format=3) == 4 and norm(q_format=0) == 4 and norm(eps=-1.0) == 4 and norm(eps=float("nan")) == 4
    assert norm(x=None) == 1 and norm(h=None) == 1 and norm(scale=None) == 1
    for k in ("ld_x", "ld_residual", "ld_h", "ld_y"):
        assert norm(**{k: 299}) == 2
    assert norm(ld_q=304) == 2 and norm(ld_s=9) == 2 and norm(q_format=2, ld_s=2) == 2 and norm(q_format=2, ld_q=288) == 2
    assert norm(x=P + 1) == 3 and norm(h=P + 2) == 3 and norm(weight=P + 2) == 3 and norm(q=P + 8) == 3 and norm(q_format=2, ld_q=300) == 3 and norm(rstd=P + 2) == 3
    assert norm(q_format=2, scale=P + 2) == 3
    assert norm(rows=0, x=None) == 0 and norm(cols=0, x=None) == 0


def grad(rows=10, cols=300, scratch=P, size=1 << 20, **kw):
    f = dict(dy=P, ld_dy=300, dy_type=0, h=P, ld_h=300, h_type=1, rstd=P, weight=P, weight_type=1, dh=P, ld_dh=300, dx=P, ld_dx=300, dweight=P, accumulate=0)
    f.update(kw)
    return b.lib().fp4q_rms_norm_bwd(ctypes.byref(b._CNormGrad(*[f[n] for n, _ in b._CNormGrad._fields_])), rows, cols, scratch, size, None)


def test_norm_backward():
    assert b.lib().fp4q_rms_norm_bwd(None, 1, 1, None, 0, None) == 1
    assert grad(rows=-1) == 2 and grad(cols=65537) == 4 and grad(rows=1 << 31) == 4
    for k in ("dy_type", "h_type", "weight_type"):
        assert grad(**{k: 3}) == 4
    for k in ("dy", "h", "dx", "rstd"):
        assert grad(**{k: None}) == 1
    for k in ("ld_dy", "ld_h", "ld_dh", "ld_dx"):
        assert grad(**{k: 299}) == 2
    for k in ("dy", "h", "dh", "dx", "rstd", "weight", "dweight"):
        assert grad(**{k: P + 1}) == 3
    assert grad(scratch=None) == 5 and grad(size=100) == 5 and grad(scratch=P + 16) == 3
    assert grad(rows=0, dweight=None, scratch=None) == 0 and grad(cols=0) == 0
    f = b.lib().fp4q_rms_norm_bwd_scratch_bytes
    assert f(-1, 5) == f(5, 0) == f(5, 65537) == 0 and f(0, 5) >= 20 and 4096 * 4 <= f(1000, 4096) <= 1000 * 4096 * 4


def spans(*s):
    return (b._CSpan * max(len(s), 1))(*[b._CSpan(*t) for t in s])


def test_clipping():
    size = b.lib().fp4q_global_norm_scratch_bytes
    good = spans((P, 10, 20, 24, 0), (P, 1, 7, 0, 1))
    call = lambda t, n=None, norm=P, scratch=P, sb=1 << 20: b.lib().fp4q_global_norm(t, len(t) if n is None else n, norm, scratch, sb, None)  # noqa: E731
    assert size(good, 2) > 0 and size(None, 0) > 0 and size(spans(*[(P, 1, 1, 1, 0)] * 451), 451) == 2 * size(good, 2)
    assert call(good, n=-1) == 2 and call(None, n=1) == 1 and call(good, norm=None) == 1 and call(good, norm=P + 2) == 3
    assert call(good, scratch=None) == 5 and call(good, sb=8) == 5 and call(good, scratch=P + 8) == 3
    bad = [((P, -1, 20, 20, 0), 2), ((P, 10, 20, 19, 0), 2), ((P, 10, 20, 20, 2), 4), ((None, 10, 20, 20, 0), 1), ((P + 1, 10, 20, 20, 0), 3), ((P + 2, 10, 20, 20, 1), 3)]
    clip = lambda t, o=None, norm=P, m=1.0, eps=1e-6: b.lib().fp4q_clip_by_norm(t, o, len(t), norm, m, eps, None)  # noqa: E731
    for s, status in bad:
        assert call(spans(s)) == status and clip(spans(s)) == status and clip(spans((P, 10, 20, 20, 0)), spans(s)) == status
    assert clip(good, spans((P, 10, 20, 24, 0), (P, 1, 8, 0, 1))) == 2
    assert clip(good, norm=None) == 1 and clip(good, m=-1.0) == 4 and clip(good, m=float("nan")) == 4 and clip(good, eps=-1.0) == 4
    assert clip(spans((None, 0, 20, 20, 0))) == 0


def test_the_binding_refuses_tensors_of_other_kinds():
    x = torch.zeros(8, 16, dtype=torch.bfloat16)
    t = b.Fp8Tensor(8, 16, torch.zeros(8, 16, dtype=torch.uint8), torch.zeros(8, 1))
    for call in (lambda: b.fp4q_fp8_quantize(x), lambda: b.fp4q_fp8_gemm_fwd(t, t), lambda: b.fp4q_fp8_gemm_dgrad(t, t), lambda: b.fp4q_fp8_gemm_wgrad(t, t), lambda: b.fp4q_rms_norm(x),
                 lambda: b.fp4q_rms_norm_bwd(x, x, torch.zeros(8)), lambda: b.fp4q_global_norm([x]), lambda: b.fp4q_clip_grad_norm([x], 1.0)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(TypeError):
        b.fp4q_rms_norm([1.0])
    with pytest.raises(TypeError):
        b.fp4q_global_norm([1.0])


def test_the_layers_refuse_shapes_that_do_not_belong_together():
    x, w, g = torch.zeros(10, 16), torch.zeros(8, 16), torch.zeros(16)
    for call in (lambda: autograd.fp8_linear(x, w[:, :8]), lambda: autograd.fp8_linear(x, g), lambda: autograd.rms_norm(x, g[:8]), lambda: autograd.rms_norm(x, g, x[:5]),
                 lambda: autograd.rms_norm_fp8_linear(x, g[:8], w), lambda: autograd.rms_norm_fp8_linear(x, g, w, x[:, :8])):
        with pytest.raises(ValueError):
            call()
    assert autograd.clip_grad_norm_([torch.nn.Parameter(g)], 1.0) == 0
