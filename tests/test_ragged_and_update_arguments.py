"""What the ragged products and the orthogonalised update refuse, without a device: the C entry points check their arguments before anything
is enqueued, the binding checks its tensors."""
import ctypes

import pytest
import torch

from paper_2607_24953_b200 import binding as b

P = 0x100000


def groups(n=2, alignment=0, offsets=P):
    return ctypes.byref(b._CGroups(n, alignment, offsets))


def fwd(x=P, T=10, K=64, ldx=64, w=P, w_rows=80, ldw=64, y=P, ldy=40, dt=0, g=None, ws=P, wsb=256):
    return b.lib().fp4q_ragged_gemm_fwd(x, T, K, ldx, w, w_rows, ldw, y, ldy, dt, g or groups(), ws, wsb, None)


def dgrad(x=P, T=10, N=40, ldx=40, w=P, w_rows=80, K=64, ldw=64, y=P, ldy=64, dt=0, g=None, ws=P, wsb=256):
    return b.lib().fp4q_ragged_gemm_dgrad(x, T, N, ldx, w, w_rows, K, ldw, y, ldy, dt, g or groups(), ws, wsb, None)


def wgrad(dy=P, T=10, N=40, ldd=40, x=P, K=64, ldx=64, dw=P, ldw=64, dt=1, accumulate=0, g=None, ws=P, wsb=256):
    return b.lib().fp4q_ragged_gemm_wgrad(dy, T, N, ldd, x, K, ldx, dw, ldw, dt, accumulate, g or groups(), None, 0, ws, wsb, None)


def test_products():
    for f in (fwd, dgrad, wgrad):
        assert f(T=-1) == 2 and f(K=-1) == 2
        assert f(ldx=32) == 2 and f(ldw=16) == 2
        assert f(dt=2) == 4 and f(dt=0x400) == 4
        assert f(g=groups(0)) == 2 and f(g=groups(-3)) == 2 and f(g=groups(2048)) == 4
        assert f(g=groups(alignment=64)) == 4 and f(g=groups(offsets=None)) == 1
        assert f(ws=None) == 5 and f(wsb=100) == 5 and f(ws=P + 16) == 3
        assert f(x=None) == 1 and f(x=P + 8) == 3
        assert f(T=1 << 31) == 4 and f(K=1 << 31, ldx=1 << 31, ldw=1 << 31, ldy=1 << 31) in (2, 4) if f is not wgrad else True
        assert f(ldx=68) == 3
    for f in (fwd, dgrad):
        assert f(w=None) == 1 and f(w=P + 2) == 3 and f(ldw=68) == 3
        assert f(y=None) == 1 and f(y=P + 8) == 3 and f(ldy=68) == 3 and f(ldy=32) == 2
        assert f(w_rows=81) == 2
        assert f(T=0, y=None, x=None) == 0                  # nothing to do
    assert fwd(w_rows=0) == 0 and dgrad(w_rows=60) == 2
    assert wgrad(dt=0, accumulate=1) == 4 and wgrad(dw=None) == 1 and wgrad(dw=P + 4) == 3 and wgrad(ldw=66) == 3 and wgrad(ldd=44) == 3
    assert wgrad(N=0, dw=None) == 0


C5 = (ctypes.c_float * 15)(*[3.4445, -4.775, 2.0315] * 5)


def test_scratch_of_weight_gradients():
    f = b.lib().fp4q_ragged_gemm_wgrad_scratch_bytes
    assert f(0, 64, 64, 1) == f(64, 0, 64, 1) == f(64, 64, 64, 0) == f(64, 64, 64, 2048) == f(-1, 64, 64, 1) == 0
    assert f(300, 1024, 512, 64) == 0                       # nothing to cut
    assert 0 < f(131072, 768, 2048, 1) < 1 << 28 and 0 < f(131072, 128, 64, 4) < 1 << 28
    call = lambda scratch, size: b.lib().fp4q_ragged_gemm_wgrad(P, 131072, 64, 64, P, 64, 64, P, 64, 1, 0, None, scratch, size, P, 256, None)
    assert call(P, 16) == 5 and call(P + 16, 1 << 30) == 3


def update(g=P, dt=1, count=2, rows=30, cols=50, ldg=50, m=P, ldm=50, eps=1e-7, c=C5, steps=5, out=P, ldo=50, scratch=P, sb=1 << 30, ws=P, wsb=256):
    return b.lib().fp4q_newton_schulz(g, dt, count, rows, cols, ldg, m, ldm, 0.9, 1, c, steps, eps, 1.0, out, ldo, scratch, sb, ws, wsb, None)


def test_updates():
    assert update(count=-1) == 2 and update(rows=-1) == 2 and update(cols=-1) == 2
    assert update(ldg=49) == 2 and update(ldm=49) == 2 and update(ldo=49) == 2
    assert update(dt=2) == 4 and update(dt=0x101) == 4
    assert update(steps=0) == 4 and update(steps=65) == 4 and update(eps=-1.0) == 4 and update(eps=float("nan")) == 4
    assert update(c=None) == 1 and update(g=None) == 1 and update(out=None) == 1
    assert update(g=P + 2) == 3 and update(m=P + 2) == 3 and update(out=P + 1) == 3
    assert update(scratch=None) == 5 and update(sb=1000) == 5 and update(scratch=P + 16) == 3
    assert update(ws=None) == 5 and update(wsb=8) == 5 and update(ws=P + 8) == 3
    assert update(rows=1 << 21, ldg=50) == 4 and update(count=70000) == 4
    assert update(count=0, g=None, out=None, scratch=None, ws=None) == 0
    for bad in ([11.0, 0.0, 0.0], [1.0, 120.0, 0.0], [float("inf"), 0.0, 0.0], [3.0, 3.0, 3.0] * 4):
        assert update(c=(ctypes.c_float * len(bad))(*bad), steps=len(bad) // 3) == 4


def test_scratch_sizes():
    f = b.lib().fp4q_newton_schulz_scratch_bytes
    assert f(0, 5, 5) == f(2, 0, 5) == f(2, 5, -1) == f(70000, 5, 5) == f(1, 1 << 21, 5) == 0
    assert f(1, 256, 256) > 5 * 256 * 256 * 2 and f(2, 768, 2048) > 2 * (3 * 768 * 2048 + 2 * 768 * 768) * 2


def test_the_binding_refuses_tensors_of_other_kinds():
    x = torch.zeros(8, 16, dtype=torch.bfloat16)
    for f in (b.fp4q_ragged_gemm_fwd, b.fp4q_ragged_gemm_dgrad, b.fp4q_ragged_gemm_wgrad):
        with pytest.raises(ValueError, match="CUDA"):
            f(x, x, None)
    with pytest.raises(ValueError, match="CUDA"):
        b.fp4q_newton_schulz(torch.zeros(8, 16))
    with pytest.raises(TypeError):
        b.fp4q_newton_schulz([1.0, 2.0])


def test_the_layer_refuses_shapes_that_do_not_belong_together():
    from paper_2607_24953_b200.autograd import ragged_linear
    x, w, offs = torch.zeros(10, 16), torch.zeros(4, 8, 16), torch.zeros(5, dtype=torch.int64)
    for bad in [(x, w, offs[:3]), (x, w, offs[None]), (x, w[0], offs), (x[0], w, offs), (x[:, :8], w, offs)]:
        with pytest.raises(ValueError):
            ragged_linear(*bad)
