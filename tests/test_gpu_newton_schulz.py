"""Orthogonalised updates against their definition in 64 bits.

Tolerance, relative and in the Frobenius norm.  The operands of a step's products are FP16, rounded by at most 2^-11 of the value, 2^-11/sqrt(3) in
the mean square.  With singular values of about 1, |b| + 2 |c| < 9 bounds what an error of A does to X', |P| < 3 what one of X does through P X, and one of P
is of P's size, so a step adds at most (9 * 2 (A is made of X twice and rounded once; half of it cancels) + 3 + 3) / 3 of that where all act together, and
the steps' errors are independent: sqrt(5) * 2^-11/sqrt(3) * sqrt(3^2 + 3^2 + 4^2) = 3.7e-3; the result's rounding to BF16 adds 2^-8/sqrt(3) =
2.3e-3, in quadrature 4.4e-3.  The momentum is two FP32 roundings."""
import math

import pytest
import torch

from paper_2607_24953_b200 import autograd, binding as b

pytestmark = pytest.mark.gpu
LIMIT = 4.4e-3


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def exact(u, coefficients=b.NEWTON_SCHULZ, eps=1e-7, scale=1.0):
    x = u.double()
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    for a, c1, c2 in coefficients:
        q = x @ x.mT
        x = a * x + (c1 * q + c2 * (q @ q)) @ x
    return scale * (x.mT if tall else x)


def close(got, want, limit=LIMIT):
    got, want = got.double(), want.double()
    if got.dim() == 2:
        got, want = got[None], want[None]
    for g, w in zip(got, want):
        assert (g - w).norm() <= limit * w.norm() + 1e-30, ((g - w).norm() / w.norm()).item()


SIZES = [(1, 1), (1, 5), (7, 1), (16, 16), (17, 300), (300, 33), (64, 64), (129, 257), (257, 129), (128, 4096), (1003, 777), (777, 1003), (520, 2048),
         (2048, 520), (2600, 1100), (1500, 2000), (4751, 63), (20, 9000), (300, 5000)]


@pytest.mark.parametrize("rows,cols", SIZES)
def test_one_matrix(rows, cols):
    ws = b.alloc_workspace("cuda")
    for dtype, scale in ((torch.float32, 1.0), (torch.bfloat16, 3.7)):
        g = randn(rows, rows, cols).to(dtype)
        out = b.fp4q_newton_schulz(g, ws=ws, scale=scale)
        assert out.shape == g.shape and out.dtype == torch.bfloat16
        close(out, exact(g, scale=scale))
        assert torch.equal(out, b.fp4q_newton_schulz(g, ws=ws, scale=scale))      # the same every time
    assert b.fp4q_workspace_status(ws) == 0


@pytest.mark.parametrize("count,rows,cols", [(3, 100, 200), (5, 200, 100), (40, 256, 512), (130, 64, 64), (1, 50, 60), (9, 768, 300), (30, 40, 1500), (85, 2382, 45)])
def test_stacks_with_and_without_momentum(count, rows, cols):
    for dtype in (torch.float32, torch.bfloat16):
        for nesterov in (True, False):
            g, m = (randn(1, count, rows, cols) * 1e-3).to(dtype), randn(2, count, rows, cols) * 4e-3
            old = m.clone()
            out = b.fp4q_newton_schulz(g, momentum=m, beta=0.9, nesterov=nesterov)
            beta = float(torch.tensor(0.9, dtype=torch.float32))
            want = beta * old.double() + g.double()
            assert ((m.double() - want).abs() <= 2 ** -23 * (old.double().abs() + g.double().abs())).all()
            close(out, exact(beta * want + g.double() if nesterov else want))


def test_matrices_of_low_rank_and_of_fast_falling_singular_values():
    for m, n, rank in ((768, 2048, 8), (768, 2048, 100), (2048, 2048, 64), (512, 300, 1), (100, 100, 3), (300, 2000, 17)):
        g = randn(1, m, rank) @ randn(2, rank, n)
        close(b.fp4q_newton_schulz(g), exact(g))
    g = (randn(3, 600, 400) * torch.logspace(0, -4, 400, device="cuda")) @ randn(4, 400, 1000)
    close(b.fp4q_newton_schulz(g), exact(g))


@pytest.mark.parametrize("factor", [1e-30, 1e-12, 1e25])
def test_gradients_of_any_size(factor):
    g = randn(1, 150, 260) * factor
    close(b.fp4q_newton_schulz(g, eps=0.0), exact(g, eps=0.0))
    small = randn(1, 150, 260) * 1e-12                     # beside eps
    close(b.fp4q_newton_schulz(small, eps=1e-9), exact(small, eps=float(torch.tensor(1e-9))))


def test_zeros_infinities_and_what_is_no_number_stay_in_their_matrix():
    for rows, cols in ((100, 300), (300, 100), (700, 600)):
        g = randn(1, 5, rows, cols)
        want = b.fp4q_newton_schulz(g)
        bad = g.clone()
        bad[1] = 0
        bad[3, 5, 7] = float("inf")
        bad[4, 0, 0] = float("nan")
        got = b.fp4q_newton_schulz(bad)
        assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
        assert not got[1].any() and got[3].isnan().all() and got[4].isnan().all()


@pytest.mark.parametrize("rows,cols", [(30, 77), (131, 67), (200, 333)])
def test_pitches_and_addresses_of_any_kind(rows, cols):
    count, want = 3, None
    for shift, pitch in ((0, cols), (1, cols + 1), (3, cols + 5), (4, (cols + 7) // 8 * 8)):
        def place(t):
            buf = torch.full((shift + count * rows * pitch + 8,), 5.0, dtype=t.dtype, device="cuda")
            view = buf[shift:shift + count * rows * pitch].view(count, rows, pitch)[:, :, :cols]
            view.copy_(t)
            return buf, view
        g, m = randn(1, count, rows, cols), randn(2, count, rows, cols)
        (_, gv), (mb, mv), (ob, ov) = place(g), place(m), place(torch.zeros(count, rows, cols, dtype=torch.bfloat16, device="cuda"))
        for dtype in (torch.float32, torch.bfloat16):
            gd = place(g.to(torch.bfloat16).to(dtype))[1]
            mv.copy_(m)
            ov.zero_()
            assert b.fp4q_newton_schulz(gd, momentum=mv, out=ov) is ov
            if want is None:
                want = ov.clone(), mv.clone()
            assert torch.equal(ov, want[0]) and torch.equal(mv, want[1])
            for buf, view in ((mb, mv), (ob, ov)):          # nothing beside the matrices
                view.fill_(5.0)
                assert (buf == 5).all()


def test_steps_and_coefficients():
    g = randn(1, 200, 300)
    for coefficients in (((1.5, -0.5, 0.0),), ((2.0, -1.5, 0.5),) * 8, ((3.4445, -4.775, 2.0315), (1.875, -1.25, 0.375), (1.875, -1.25, 0.375))):
        close(b.fp4q_newton_schulz(g, coefficients=coefficients), exact(g, coefficients))
    for coefficients in (((30.0, 0.0, 0.0),), ((1.0, 200.0, 0.0),), ((float("nan"), 0.0, 0.0),), ((1.5, -0.5, 0.0),) * 65):
        with pytest.raises(b.Fp4qError) as err:
            b.fp4q_newton_schulz(g, coefficients=coefficients)
        assert err.value.status == 4


def test_empty_stacks():
    for shape in ((0, 20, 30), (2, 0, 30), (2, 30, 0), (0, 5), (5, 0)):
        g = torch.zeros(*shape, device="cuda")
        assert b.fp4q_newton_schulz(g, momentum=g.clone()).shape == g.shape


def test_captured_and_on_another_stream():
    g, m = randn(1, 4, 200, 150), randn(2, 4, 200, 150)
    scratch, ws = b.alloc_newton_schulz_scratch(4, 200, 150, "cuda"), b.alloc_workspace("cuda")
    m1, m2, m3 = m.clone(), m.clone(), m.clone()
    eager = [b.fp4q_newton_schulz(g, momentum=m1, scratch=scratch, ws=ws) for _ in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = [b.fp4q_newton_schulz(g, momentum=m2, scratch=scratch, ws=ws, stream=side) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = b.fp4q_newton_schulz(g, momentum=m3, scratch=scratch, ws=ws)
    for i in range(3):
        scratch.fill_(255)                                  # nothing is kept there
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured, eager[i]) and torch.equal(other[i], eager[i])
    assert torch.equal(m1, m2) and torch.equal(m1, m3) and b.fp4q_workspace_status(ws) == 0


@pytest.mark.parametrize("count,rows,cols", [(1, 100, 200), (1, 500, 700), (3, 1000, 300), (1, 2100, 2300)])
def test_a_wait_that_runs_out_is_reported(count, rows, cols):
    g, ws = randn(1, count, rows, cols), b.alloc_workspace("cuda")
    want = b.fp4q_newton_schulz(g, ws=ws)
    b.fp4q_workspace_set_wait_limit(ws, 2000)
    b.fp4q_debug_withhold_load(ws, 1)
    b.fp4q_newton_schulz(g, ws=ws)
    assert b.fp4q_workspace_status(ws) == 7
    b.fp4q_debug_withhold_load(ws, 0)
    b.fp4q_workspace_set_wait_limit(ws, 0)
    assert torch.equal(b.fp4q_newton_schulz(g, ws=ws), want) and b.fp4q_workspace_status(ws) == 0


@pytest.mark.parametrize("count,side,other", [(1, 384, 384), (1, 385, 385), (1, 60, 3000), (2, 200, 5000), (5, 380, 1500), (1, 768, 768), (3, 640, 2000), (2, 1100, 1100)])
def test_tiles_of_every_edge_wide_and_tall(count, side, other):
    g = randn(1, count, side, other)
    close(b.fp4q_newton_schulz(g), exact(g))
    close(b.fp4q_newton_schulz(g.transpose(1, 2).contiguous()), exact(g.transpose(1, 2).contiguous()))


def test_a_training_step_of_an_expert_layer():
    # ragged products forward and backward, the update, the new master weights into FP4 and through the framework's own product
    E, n, k, T = 4, 256, 128, 700
    offs = torch.tensor([0, 100, 100, 421, 700], device="cuda")
    w = torch.nn.Parameter(randn(1, E, n, k) * 0.05)
    x, ws = randn(2, T, k).to(torch.bfloat16), b.alloc_workspace("cuda")
    m, scratch = torch.zeros_like(w), b.alloc_newton_schulz_scratch(E, n, k, "cuda")
    for step in range(3):
        w.grad = None
        y = autograd.ragged_linear(x, w, offs, ws)
        dy = (y.float() * 1e-2).to(torch.bfloat16)
        y.backward(dy)
        before, m0 = w.detach().clone(), m.clone()
        wb = before.bfloat16().double()
        grad = torch.stack([dy[i:j].double().T @ x[i:j].double() for i, j in ((0, 100), (100, 100), (100, 421), (421, 700))])
        assert (w.grad.double() - grad).norm() <= 1e-6 * grad.norm() and not w.grad[1].any()
        o = b.fp4q_newton_schulz(w.grad, momentum=m, scale=0.2 * math.sqrt(n), scratch=scratch, ws=ws)
        beta = float(torch.tensor(0.95))
        u = beta * (beta * m0.double() + w.grad.double()) + w.grad.double()
        close(o[[0, 2, 3]], exact(u, scale=0.2 * math.sqrt(n))[[0, 2, 3]])
        assert not o[1].any()
        with torch.no_grad():
            w.mul_(1 - 0.01 * 0.1).add_(o, alpha=-0.01)
        assert torch.equal(w[1], (before * (1 - 0.01 * 0.1))[1])
    qw, qx = b.fp4q_quantize2d(w.detach()[2].to(torch.bfloat16).contiguous()), b.fp4q_quantize2d(x)
    y4, y16 = b.fp4q_gemm_fwd(qx, qw, ws=ws).double(), x.double() @ w.detach()[2].double().T
    assert (y4 - y16).norm() <= 0.5 * y16.norm() and b.fp4q_workspace_status(ws) == 0
