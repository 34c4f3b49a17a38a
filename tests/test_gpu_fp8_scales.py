"""8-bit products whose scales' products leave FP32's normal range, where what they stand for does not: blocks of zeros beside small ones, tiny and huge operands, all of them in one tile.

Tolerance: that of the products (test_gpu_fp8_blocks.py: the tensor cores' 4 * 2^-22 of the absolute products S of a block, two roundings a block and one of the scales' product) with one rounding more for a
block's product, which is multiplied in two steps where the scales are large.  A product of scales below FP32's normal range is off by 2^-150, a block's share of a sum, |x| < 2^25 of these, by 2^-125."""
import pytest
import torch

from paper_2607_24953_b200 import binding as b

pytestmark = pytest.mark.gpu
LEAST = 2.0 ** -100 / 448


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def codes(seed, rows, cols, most=0x7E):
    q = torch.randint(0, most + 1, (rows, cols), generator=gen(seed), device="cuda") | torch.randint(0, 2, (rows, cols), generator=gen(seed + 1), device="cuda") * 128
    return q.to(torch.uint8)


def powers(seed, shape, lo, hi):
    """Numbers of all mantissas from 2^lo to 2^hi."""
    e = torch.rand(shape, generator=gen(seed), device="cuda", dtype=torch.float64) * (hi - lo) + lo
    return torch.exp2(e).float()


def pick(seed, shape, share):
    return torch.rand(shape, generator=gen(seed), device="cuda") < share


def blocks(n):
    return (n + 127) // 128


def wide(scale, down, rows, cols):
    return scale.repeat_interleave(down, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def clear(q, scale_mask, down):
    """No codes in the blocks of scale_mask."""
    q[wide(scale_mask, down, *q.shape)] = 0


# Each: codes and scales of both operands, A in 1D blocks, B in blocks of `down` rows.
def tiny(m, n, k, down):
    return codes(1, m, k), powers(3, (m, blocks(k)), -80, -60), codes(5, n, k), powers(7, (-(-n // down), blocks(k)), -75, -62)


def zeros_beside_small(m, n, k, down):
    a, w = codes(1, m, k), codes(5, n, k)
    sa, sw = powers(3, (m, blocks(k)), -36, -26), powers(7, (-(-n // down), blocks(k)), -36, -8)
    for q, s, d, seed in ((a, sa, 1, 11), (w, sw, down, 13)):
        none = pick(seed, s.shape, 0.3)
        clear(q, none, d)
        s[none | pick(seed + 1, s.shape, 0.05)] = LEAST          # and some blocks of numbers below 2^-100
    return a, sa, w, sw


def all_sizes(m, n, k, down):
    a, w = codes(1, m, k), codes(5, n, k)
    sa, sw = powers(3, (m, blocks(k)), -109, 2), powers(7, (-(-n // down), blocks(k)), -109, 20)
    huge_a, huge_w = pick(11, sa.shape, 0.1), pick(13, sw.shape, 0.2)
    sa[huge_a], sw[huge_w] = powers(15, sa.shape, 60, 119)[huge_a], powers(17, sw.shape, 60, 119)[huge_w]
    clear(a, huge_a, 1)
    clear(w, huge_w, down)
    return a, sa, w, sw


def huge_scales_of_tiny_codes(m, n, k, down):
    a, w = codes(1, m, k, 1), codes(5, n, k, 1)                  # 0 and 2^-9
    sa, sw = powers(3, (m, blocks(k)), 66, 68), powers(7, (-(-n // down), blocks(k)), 60, 66)
    return a, sa, w, sw


def check(y, a, sa, w, sw, down, k):
    x = a.view(torch.float8_e4m3fn).double() * wide(sa, 1, a.shape[0], k).double()
    v = w.view(torch.float8_e4m3fn).double() * wide(sw, down, w.shape[0], k).double()
    want, s = x @ v.T, x.abs() @ v.abs().T
    nb = blocks(k)
    tol = s * (4 * 2.0 ** -22 + (nb + 4) * 2.0 ** -24) + nb * 2.0 ** -125
    inside = s < 3e38                                            # no sum on the way to the result can overflow
    assert inside.any()
    off = (y.double() - want).abs()
    assert (off <= tol)[inside].all(), float((off / tol)[inside].max())
    return want, s


def padded(q):
    buf = torch.zeros(q.shape[0], (q.shape[1] + 15) // 16 * 16, dtype=torch.uint8, device="cuda")
    buf[:, :q.shape[1]] = q
    return buf


CASES = [tiny, zeros_beside_small, all_sizes, huge_scales_of_tiny_codes]
SHAPES = [(1, 300, 700), (3, 130, 4096), (20, 1000, 1500), (50, 257, 640), (64, 128, 128), (200, 256, 2731), (129, 1003, 100), (1024, 2048, 2048), (2048, 2048, 2048), (2300, 2148, 1111), (4000, 2000, 300)]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_one_operand_in_square_blocks(m, n, k, case):
    a, sa, w, sw = case(m, n, k, 128)
    ws = b.alloc_workspace("cuda")
    y = b.fp4q_fp8_gemm_fwd(b.Fp8Tensor(m, k, padded(a), sa), b.Fp8Tensor(n, k, padded(w), sw, square=True), dt=b.OUT_F32, ws=ws)
    check(y, a, sa, w, sw, 128, k)
    # the same product as an input gradient: the codes of the transpose, the scales where they are
    y2 = b.fp4q_fp8_gemm_dgrad(b.Fp8Tensor(m, k, padded(a), sa), b.Fp8Tensor(k, n, None, sw.T.contiguous(), padded(w), None, True), dt=b.OUT_F32, ws=ws)
    assert torch.equal(y.view(torch.int32) if y.is_contiguous() else y.contiguous().view(torch.int32), y2.contiguous().view(torch.int32))
    assert b.fp4q_workspace_status(ws) == 0


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("m,n,k", [(40, 60, 100), (256, 256, 4000), (300, 128, 3001), (1003, 731, 515), (2048, 1024, 1000), (2048, 2048, 2048), (2304, 2200, 700), (3000, 2148, 300)])
def test_both_operands_in_1d_blocks(m, n, k, case):
    a, sa, w, sw = case(m, n, k, 1)
    ws = b.alloc_workspace("cuda")
    A, W = b.Fp8Tensor(k, m, None, None, padded(a), sa), b.Fp8Tensor(k, n, None, None, padded(w), sw)
    check(b.fp4q_fp8_gemm_wgrad(A, W, ws=ws), a, sa, w, sw, 1, k)
    assert b.fp4q_workspace_status(ws) == 0


@pytest.mark.parametrize("rows", [8, 100, 2048])
def test_scales_of_zero_and_of_either_sign(rows):
    a, sa, w, sw = zeros_beside_small(rows, 512, 640, 128)
    sa[:, 1] = 0
    sa[::3, 2] *= -1
    sw[1] *= -1
    y = b.fp4q_fp8_gemm_fwd(b.Fp8Tensor(rows, 640, padded(a), sa), b.Fp8Tensor(512, 640, padded(w), sw, square=True), dt=b.OUT_F32)
    check(y, a, sa, w, sw, 128, 640)


def test_layers_of_tiny_numbers():
    # From the quantizer: activations of 2^-60 and weights of 2^-60, with rows and columns of zeros.
    x, w = torch.randn(300, 520, generator=gen(1), device="cuda") * 2.0 ** -60, torch.randn(384, 520, generator=gen(2), device="cuda") * 2.0 ** -60
    x[:128], w[128:256] = 0, 0
    X, W = b.fp4q_fp8_quantize(x), b.fp4q_fp8_quantize(w, square=True)
    y = b.fp4q_fp8_gemm_fwd(X, W, dt=b.OUT_F32)
    check(y, X.q[:, :520].contiguous(), X.scale, W.q[:, :520].contiguous(), W.scale, 128, 520)
    assert not y[:128].any() and not y[:, 128:256].any()


@pytest.mark.parametrize("rows", [5, 200, 2048])
def test_infinities_that_are_none_of_the_scales(rows):
    # A product that is too large for FP32, and codes that are NaN, stay what they are beside large scales.
    a, sa, w, sw = all_sizes(rows, 512, 640, 128)
    a[1, 3], a[2, :128], w[100, :128] = 0x7F, 0x78, 0x78          # NaN; 128 times 256
    sa[2, 0], sw[0, 0] = 2.0 ** 100, 2.0 ** 100
    y = b.fp4q_fp8_gemm_fwd(b.Fp8Tensor(rows, 640, padded(a), sa), b.Fp8Tensor(512, 640, padded(w), sw, square=True), dt=b.OUT_F32)
    assert y[1].isnan().all() and y[2, 100] == float("inf")
    a[1, 3] = 0
    check(y[3:], a[3:], sa[3:], w, sw, 128, 640)


def test_accumulating_beside_large_scales():
    for m, n, k in ((256, 256, 4000), (2048, 2048, 512)):
        a, sa, w, sw = all_sizes(m, n, k, 1)
        A, W = b.Fp8Tensor(k, m, None, None, padded(a), sa), b.Fp8Tensor(k, n, None, None, padded(w), sw)
        once = b.fp4q_fp8_gemm_wgrad(A, W)
        before = torch.randn(m, n, generator=gen(30), device="cuda")
        out = before.clone()
        b.fp4q_fp8_gemm_wgrad(A, W, out=out, accumulate=True)
        assert torch.equal(out, before + once)
