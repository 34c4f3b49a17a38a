"""Where orthogonalised updates are exact, or closer to their definition than one FP16 operand would be."""
import math

import pytest
import torch

from paper_2607_24953_b200 import binding as b

pytestmark = pytest.mark.gpu


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def exact(u, coefficients=b.NEWTON_SCHULZ, eps=1e-7):
    x = u.double()
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    for a, c1, c2 in coefficients:
        q = x @ x.mT
        x = a * x + (c1 * q + c2 * (q @ q)) @ x
    return x.mT if tall else x


@pytest.mark.parametrize("count,side,other", [(1, 500, 700), (5, 400, 600), (1, 1300, 1400), (12, 800, 900)])
def test_the_polynomials_diagonal_is_rounded_once(count, side, other):
    # One row of 256 elements +-1/16 in each matrix: X, A = e e^T and a + b A are exact in FP16 (a = 20 and b = -19.3046875 make 89/128 = 356/512), and so
    # is the result in BF16; b A alone, 9884/512, is none of FP16's numbers.
    g = torch.zeros(count, side, other, device="cuda")
    for i in range(count):
        at = torch.randperm(other, generator=torch.Generator().manual_seed(i))[:256].cuda()
        g[i, (77 + 131 * i) % side, at] = torch.sign(randn(i, 256)) * 3.0
    want = (torch.sign(g) * (89 / 128 / 16)).to(torch.bfloat16)
    step = ((20.0, -19.3046875, 0.0),)
    assert torch.equal(b.fp4q_newton_schulz(g, coefficients=step, eps=0.0), want)
    assert torch.equal(b.fp4q_newton_schulz(g.mT.contiguous(), coefficients=step, eps=0.0), want.mT)


@pytest.mark.parametrize("side,other", [(385, 8000), (500, 5000), (640, 640)])
def test_products_that_are_little_but_their_diagonals(side, other):
    # Operands in one FP16 number, rounded by 2^-11 / sqrt(3) in the mean square, independently from row to row as the diagonals differ.  Per step 9 times
    # that for A (at most |b| + 2 |c|) and 3 for P and for X, in quadrature over five steps 6.3e-3 where all of it acts; A's error is one of the diagonal
    # alone and meets b + 2 c A instead of |b| + 2 |c|, below 5: sqrt(5 (5^2 + 3^2 + 3^2)) 2^-11 / sqrt(3) = 4.1e-3.  The result's rounding: 2^-8 / sqrt(3).
    g = randn(1, side, other) if side != other else torch.diag(1 + torch.rand(side, generator=torch.Generator("cuda").manual_seed(2), device="cuda"))
    for u in (g, g.T.contiguous()):
        want = exact(u)
        assert (b.fp4q_newton_schulz(u).double() - want).norm() <= math.hypot(4.1e-3, 2 ** -8 / 3 ** 0.5) * want.norm()


@pytest.mark.parametrize("count,cols", [(4, 50), (3, 700)])
def test_stacks_of_single_rows_in_any_pitch(count, cols):
    # As first rows of larger matrices, or as a padded matrix's rows: one step of (1.5, -0.5, 0) leaves a row of length 1 as it is.
    big, m, out = randn(1, count, 6, cols + 14), torch.zeros(count, 5, cols, device="cuda"), torch.zeros(count, 3, cols + 3, dtype=torch.bfloat16, device="cuda")
    step = ((1.5, -0.5, 0.0),)
    rows = big[:, 0, :cols]
    want = b.fp4q_newton_schulz(rows.contiguous().view(count, 1, cols), coefficients=step)
    assert torch.equal(b.fp4q_newton_schulz(big[:, :1, :cols], coefficients=step), want)
    assert torch.equal(b.fp4q_newton_schulz(rows.unsqueeze(1), coefficients=step), want)
    o = out[:, 1:2, :cols]
    assert b.fp4q_newton_schulz(big[:, :1, :cols], momentum=m[:, 2:3], coefficients=step, out=o) is o
    # 2^-8 of the value for BF16, and 2^-20 for sums and products in 22 bits
    assert ((o.double() - rows.double()[:, None] / rows.double().norm(dim=1)[:, None, None]).abs() <= (2 ** -8 + 2 ** -20) * o.double().abs() + 1e-7).all()
    assert torch.equal(m[:, 2], rows) and not m[:, :2].any() and not m[:, 3:].any()
    assert not out[:, 0].any() and not out[:, 2].any() and not out[:, :, cols:].any()
    with pytest.raises(b.Fp4qError):
        b.fp4q_newton_schulz(big[:1, :1, :cols].expand(count, 1, cols), momentum=m[:1, :1].expand(count, 1, cols))       # rows that lie in one another


@pytest.mark.parametrize("count,rows,cols", [(1, 768, 2048), (1, 200, 300), (1, 2048, 520), (6, 300, 70), (5, 900, 800), (40, 300, 400)])
@pytest.mark.parametrize("below", [0.7, 1e-2, 1e-5, 1e-7, 1e-9, 1e-14, 1e-18])
def test_norms_far_below_eps(count, rows, cols, below):
    # Each matrix in its own distance from eps, one of them above it, one of zeros.  The limit is that of norms above eps: operands in FP16 in the mean
    # square, 2^-11 / sqrt(3) sqrt(5 (3^2 + 3^2 + 4^2)), and BF16's rounding, 2^-8 / sqrt(3).
    eps = float(torch.tensor(1e-7))
    g = randn(1, count, rows, cols)
    factors = [below * 0.31 ** (i % 5) for i in range(count)]
    if count > 3:
        factors[1], factors[2] = 1e9, 0.0
    g *= (torch.tensor(factors, device="cuda", dtype=torch.float64) * eps / g.double().norm(dim=(1, 2))).float()[:, None, None]
    for coefficients in (b.NEWTON_SCHULZ, ((2.0, -1.5, 0.5),) * 5, ((9.0, -9.0, 0.0), (0.5, 0.0, 0.0), (1.5, -0.5, 0.0))):
        got, want = b.fp4q_newton_schulz(g, coefficients=coefficients, eps=eps).double(), exact(g, coefficients, eps)
        for i in range(count):
            assert (got[i] - want[i]).norm() <= 4.4e-3 * want[i].norm(), (i, factors[i])


@pytest.mark.parametrize("count,rows,cols", [(1, 5, 7), (1, 16, 16), (1, 20, 20), (1, 64, 64), (1, 100, 64), (2, 64, 128), (1, 128, 120), (30, 64, 64), (130, 64, 64), (200, 128, 128),
                                             (150, 70, 128), (150, 128, 70), (1, 17, 300), (1, 300, 33), (1, 129, 257), (40, 256, 256), (100, 256, 200), (1, 384, 384), (80, 384, 300)])
def test_short_sides_compute_with_both_parts_of_their_operands(count, rows, cols):
    # What is beyond BF16's rounding, half a step of the result at most.  In units of 2^-22: an operand's two parts are off by 1, the product of the lower
    # ones, left out, is 1, the cut-off of K / 16 instructions 1 each, and the new value's two parts 1: 4 + K / 16 a product.  A's counts 2 (|b| + 2 |c|) = 18
    # times at most, half of which cancels, P's and X's 3 each, in a result of 3: 8 a step, 5 steps.  Without one of the lower parts an operand is off by 2^11 units.
    g = randn(rows + count, count, rows, cols)
    got, want = b.fp4q_newton_schulz(g).double(), exact(g)
    half = torch.ldexp(torch.full_like(got, 2.0 ** -8), torch.floor(torch.log2(got.abs().clamp_min(1e-300))))
    beyond = ((got - want).abs() - half).clamp_min(0.0)
    assert (beyond.norm(dim=(1, 2)) <= 40 * 2 ** -22 * (4 + max(rows, cols) / 16) * want.norm(dim=(1, 2))).all()


def test_more_than_2_to_the_31_elements():
    # The last matrices of a stack, wide and tall, whose offsets pass 32 bits; BF16 gradients, without a momentum and with one.
    for rows, cols in ((16, 1 << 20), (1 << 20, 16)):
        count = 130
        g = torch.empty(count, rows, cols, dtype=torch.bfloat16, device="cuda")
        g.normal_(generator=torch.Generator("cuda").manual_seed(1))
        out = b.fp4q_newton_schulz(g)
        for i in (0, 63, 64, 127, 128, 129):
            want = exact(g[i])
            assert (out[i].double() - want).norm() <= 4.4e-3 * want.norm()
        m = torch.ones(count, rows, cols, device="cuda")
        b.fp4q_newton_schulz(g, momentum=m, beta=0.5, nesterov=False, out=out)
        for i in (0, 128, 129):
            u = 0.5 + g[i].double()
            assert ((m[i].double() - u).abs() <= 2 ** -24 * u.abs()).all()
            want = exact(u)
            assert (out[i].double() - want).norm() <= 4.4e-3 * want.norm()
        del g, m, out
        torch.cuda.empty_cache()


@pytest.mark.parametrize("count,side,other", [(1, 24, 300_000), (3, 200, 120_000), (1, 500, 200_000), (160, 16, 70_000)])
def test_long_sides_do_not_add_up_what_the_accumulators_cut_off(count, side, other):
    # An instruction's cut-off is below 2^-22 of what all products add up to so far: with 32768 elements in an accumulator, 2048 instructions and a sum that
    # grows evenly, A's diagonal is off by 1024 * 2^-22 = 2.4e-4 at most (with 300 000 elements by 2.2e-3), and counts |b + 2 c A| < 5 times a step at
    # most: as independent steps 5 sqrt(5) 2.4e-4 = 2.7e-3 beside the limit for shorter sides, 4.4e-3 above a side of 384 and BF16's rounding below.
    g = randn(1, count, side, other) * torch.exp(0.5 * randn(2, count, side, 1))           # rows of several lengths: their roundings are independent
    limit = math.hypot(2.7e-3, 2 ** -8 / 3 ** 0.5 if side <= 384 else 4.4e-3)
    for u in (g, g.mT.contiguous()):
        got = b.fp4q_newton_schulz(u).double()
        for i in range(0, count, 53):
            want = exact(u[i])
            assert (got[i] - want).norm() <= limit * want.norm()


@pytest.mark.parametrize("rows,cols", [(40, 60), (500, 700)])
def test_zeros_beside_the_smallest_eps(rows, cols):
    for eps in (1e-45, 1e-38, 1e-30, 1e-7, 1.0):
        g = torch.zeros(3, rows, cols, device="cuda")
        g[1] = randn(1, rows, cols)
        out = b.fp4q_newton_schulz(g, eps=eps)
        assert not out[0].any() and not out[2].any()
        want = exact(g[1], eps=float(torch.tensor(eps)))
        assert (out[1].double() - want).norm() <= 4.4e-3 * want.norm()
