"""8-bit tensors with a scale for every block of 128: the quantizer bit for bit against the definition in FP32 torch operations, the products against 64-bit sums.

Tolerance of the products: the tensor cores add 32 products to an accumulator at a time and cut the sum off at 2^-22 of its largest term at worst, so the four instructions of a block are
off by at most 4 * 2^-22 of the block's absolute products; every block adds two roundings (its scales, its sum) of 2^-24, and the scales' product one.  With S the sum of the absolute
products over the whole contraction in b blocks that is S (4 * 2^-22 + (b + 3) 2^-24); a BF16 output adds half a step, 2^-8 of the result at most (2^-9 relative to the step)."""
import pytest
import torch

from paper_2607_24953_b200 import binding as b

pytestmark = pytest.mark.gpu
TOP, LEAST = 448.0, 2.0 ** -100


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def codes(x, down):
    """(bytes, scales) by the definition, one FP32 operation after the other.  (torch divides by a number as it multiplies by its rounded reciprocal; a quotient of FP32 numbers in 64 bits,
    rounded to FP32, is the FP32 quotient.)"""
    r, c = x.shape
    f = torch.nn.functional.pad(x.float(), (0, -c % 128, 0, -r % down)).reshape(-(-r // down), down, -(-c // 128), 128)
    m = torch.where(f.isfinite(), f.abs(), 0.0).amax((1, 3), keepdim=True).clamp_min(LEAST)
    v = f * (TOP / m.double()).float()
    v = torch.where(f.isinf(), float("nan"), v).clamp(-TOP, TOP)
    q = v.to(torch.float8_e4m3fn).view(torch.uint8)
    q = torch.where(f.isnan() | f.isinf(), 0x7F, q)
    return q.reshape(q.shape[0] * down, -1)[:r, :c], (m.double() / TOP).float()[:, 0, :, 0]


def check_quantizer(x, square, **kw):
    t = b.fp4q_fp8_quantize(x, square=square, **kw)
    r, c = x.shape
    want, scale = codes(x, 128 if square else 1)
    if t.q is not None:
        assert torch.equal(t.q[:, :c], want)
        assert not t.q[:, c:(c + 15) // 16 * 16].any()
    if t.scale is not None:
        assert torch.equal(t.scale[:, :scale.shape[1]], scale)
    if t.q_t is not None:
        want_t, scale_t = (want.T, None) if square else codes(x.T, 1)
        assert torch.equal(t.q_t[:, :r], want_t)
        assert not t.q_t[:, r:(r + 15) // 16 * 16].any()
        if not square:
            assert torch.equal(t.scale_t[:, :scale_t.shape[1]], scale_t)
    return t


SIZES = [(1, 1), (1, 4096), (5, 129), (128, 128), (127, 255), (300, 777), (1000, 16), (2, 2731), (513, 640)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("r,c", SIZES)
def test_quantizer(r, c, square, dtype):
    check_quantizer((randn(r + c, r, c) * torch.exp(3 * randn(7, r, 1))).to(dtype), square)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pitch,start", [(8, 0), (777, 1), (801, 3), (1001, 6), (784, 8)])
def test_quantizer_of_rows_that_start_anywhere(dtype, pitch, start):
    cols = min(pitch, 770)
    buf = randn(1, 70 * pitch + 16).to(dtype)
    x = buf[start:start + 69 * pitch + cols].as_strided((70, cols), (pitch, 1))
    for square in (False, True):
        check_quantizer(x, square)


def test_quantizer_of_one_orientation_into_buffers_of_the_callers():
    x = randn(3, 200, 300).to(torch.bfloat16)
    for want, want_t in ((True, False), (False, True)):
        for square in (False, True):
            t = check_quantizer(x, square, want=want, want_t=want_t)
            assert (t.q is None) != want and (t.q_t is None) != want_t
            out = b.alloc_fp8tensor(200, 300, "cuda", square, want, want_t)
            assert b.fp4q_fp8_quantize(x, out=out, square=square) is out
            for name in ("q", "scale", "q_t", "scale_t"):
                p, q = getattr(t, name), getattr(out, name)
                assert (p is None) == (q is None)
                n = {"q": 300, "q_t": 200}.get(name)
                assert p is None or torch.equal(p[:, :n], q[:, :n])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantizer_of_zeros_infinities_nan_and_tiny_and_huge_numbers(dtype):
    x = randn(5, 260, 390)
    x[0] = 0
    x[3] *= 1e-36
    x[4] *= 1e-30
    x[5] *= 1e37
    x[7, 5], x[8, 200], x[8, 201] = float("inf"), float("nan"), float("-inf")
    x[200:, 256:] = 0
    x[9, :128] = float("inf")
    for square in (False, True):
        check_quantizer(x.to(dtype), square)


def test_quantizer_leaves_what_lies_behind_its_rows():
    x = randn(2, 40, 100).to(torch.bfloat16)
    q, s = torch.full((40, 160), 9, dtype=torch.uint8, device="cuda"), torch.full((40, 4), 9.0, device="cuda")
    b.fp4q_fp8_quantize(x, out=b.Fp8Tensor(40, 100, q, s))
    assert (q[:, 112:] == 9).all() and (s[:, 1:] == 9).all()


def values(q, scale, down):
    r, c = q.shape
    return q.view(torch.float8_e4m3fn).double() * scale.double().repeat_interleave(down, 0)[:r].repeat_interleave(128, 1)[:, :c]


def check_product(y, a, w, before=None):
    want, s = a @ w.T, a.abs() @ w.abs().T
    blocks = -(-a.shape[1] // 128)
    tol = s * (4 * 2.0 ** -22 + (blocks + 3) * 2.0 ** -24)
    if before is not None:
        want = want + before.double()
        tol = tol + (want.abs() + tol) * 2.0 ** -24
    if y.dtype == torch.bfloat16:
        tol = tol + (want.abs() + tol) * 2.0 ** -8
    off = (y.double() - want).abs()
    assert (off <= tol).all(), float((off / tol.clamp_min(1e-300)).max())


def operands(t, n, k, seed=0):
    x = (randn(seed, t, k) * torch.exp(randn(seed + 1, t, 1))).to(torch.bfloat16)
    w = randn(seed + 2, n, k) * 0.02
    dy = (randn(seed + 3, t, n) * torch.exp(2 * randn(seed + 4, t, 1))).to(torch.bfloat16)
    return b.fp4q_fp8_quantize(x), b.fp4q_fp8_quantize(w, square=True), b.fp4q_fp8_quantize(dy)


def check_all(t, n, k, dt, ws):
    X, W, dY = operands(t, n, k)
    x, w, dy = values(X.q[:, :k], X.scale, 1), values(W.q[:, :k], W.scale, 128), values(dY.q[:, :n], dY.scale, 1)
    xt, dyt = values(X.q_t[:, :t], X.scale_t, 1), values(dY.q_t[:, :t], dY.scale_t, 1)
    check_product(b.fp4q_fp8_gemm_fwd(X, W, dt=dt, ws=ws), x, w)
    check_product(b.fp4q_fp8_gemm_dgrad(dY, W, dt=dt, ws=ws), dy, w.T)
    dw = b.fp4q_fp8_gemm_wgrad(dY, X, dt=dt, ws=ws)
    check_product(dw, dyt, xt)
    if dt == b.OUT_F32:
        before = randn(9, n, (k + 3) // 4 * 4)[:, :k]
        acc = before.clone() if k % 4 == 0 else torch.empty(n, (k + 3) // 4 * 4, device="cuda")[:, :k].copy_(before)
        check_product(b.fp4q_fp8_gemm_wgrad(dY, X, out=acc, dt=dt, accumulate=True, ws=ws), dyt, xt, before)
    assert b.fp4q_workspace_status(ws) == 0


SHAPES = [(1, 1, 1), (1, 4096, 2048), (2, 130, 300), (7, 1000, 128), (16, 256, 4096), (17, 2731, 500), (33, 300, 1003), (64, 640, 640), (65, 129, 257), (128, 256, 256),
          (300, 520, 544), (1, 11008, 16), (1999, 1003, 731), (512, 1024, 4096), (2048, 768, 2048), (4096, 128, 100)]


@pytest.mark.parametrize("dt", [b.OUT_BF16, b.OUT_F32])
@pytest.mark.parametrize("t,n,k", SHAPES)
def test_products(t, n, k, dt):
    check_all(t, n, k, dt, b.alloc_workspace("cuda"))


@pytest.mark.parametrize("t,n,k", [(8192, 2048, 2048), (2500, 5632, 2048), (16384, 520, 384)])
def test_large_products(t, n, k):
    check_all(t, n, k, b.OUT_F32, b.alloc_workspace("cuda"))


@pytest.mark.parametrize("t", [3, 100])
def test_an_empty_contraction_gives_zeros(t):
    X, W = b.Fp8Tensor(t, 0, torch.empty(t, 16, dtype=torch.uint8, device="cuda")[:, :0], torch.empty(t, 0, device="cuda")), None
    W = b.Fp8Tensor(50, 0, torch.empty(50, 16, dtype=torch.uint8, device="cuda")[:, :0], torch.empty(1, 0, device="cuda"), square=True)
    for dt in (b.OUT_BF16, b.OUT_F32):
        y = torch.ones(t, 56, dtype=torch.float32 if dt else torch.bfloat16, device="cuda")
        b.fp4q_fp8_gemm_fwd(X, W, out=y[:, :50], dt=dt)
        assert not y[:, :50].any() and (y[:, 50:] == 1).all()
    d = b.Fp8Tensor(0, 40, None, None, torch.empty(40, 16, dtype=torch.uint8, device="cuda")[:, :0], torch.empty(40, 0, device="cuda"))
    dw = torch.ones(40, 40, device="cuda")
    b.fp4q_fp8_gemm_wgrad(d, d, out=dw, dt=b.OUT_F32, accumulate=True)
    assert (dw == 1).all()
    assert not b.fp4q_fp8_gemm_wgrad(d, d).any()


@pytest.mark.parametrize("t,n", [(5, 77), (40, 1003), (200, 333), (2000, 2731)])
@pytest.mark.parametrize("dt", [b.OUT_BF16, b.OUT_F32])
def test_nothing_is_written_beside_the_result(t, n, dt):
    X, W, _ = operands(t, n, 300)
    ld = (n + 7) // 8 * 8 + 16
    y = torch.full((t + 2, ld), 7.0, dtype=torch.float32 if dt else torch.bfloat16, device="cuda")
    b.fp4q_fp8_gemm_fwd(X, W, out=y[:t, :n], dt=dt)
    assert (y[:t, n:] == 7).all() and (y[t:] == 7).all()


def test_nan_in_an_operand_reaches_its_row_and_column_alone():
    x, w = randn(1, 300, 500).to(torch.bfloat16), randn(2, 400, 500)
    x[7, 3], w[300, 499] = float("nan"), float("inf")
    y = b.fp4q_fp8_gemm_fwd(b.fp4q_fp8_quantize(x), b.fp4q_fp8_quantize(w, square=True))
    bad = torch.zeros(300, 400, dtype=torch.bool, device="cuda")
    bad[7], bad[:, 300] = True, True
    assert torch.equal(y.isnan(), bad)


def test_results_do_not_depend_on_the_run():
    for t, n, k in ((1, 512, 4096), (300, 256, 4096), (3000, 1000, 1000)):
        X, W, dY = operands(t, n, k)
        first = [b.fp4q_fp8_gemm_fwd(X, W, dt=b.OUT_F32), b.fp4q_fp8_gemm_wgrad(dY, X)]
        for _ in range(5):
            again = [b.fp4q_fp8_gemm_fwd(X, W, dt=b.OUT_F32), b.fp4q_fp8_gemm_wgrad(dY, X)]
            assert all(torch.equal(p, q) for p, q in zip(first, again))


def test_a_wait_that_runs_out_is_reported():
    for t in (4, 200, 1024, 2048):                             # a kernel each
        X, W, _ = operands(t, 2048, 2048)
        ws = b.alloc_workspace("cuda")
        want = b.fp4q_fp8_gemm_fwd(X, W, ws=ws)
        b.fp4q_workspace_set_wait_limit(ws, 2000)
        b.fp4q_debug_withhold_load(ws, 1)
        b.fp4q_fp8_gemm_fwd(X, W, ws=ws)
        assert b.fp4q_workspace_status(ws) == 7
        b.fp4q_debug_withhold_load(ws, 0)
        b.fp4q_workspace_set_wait_limit(ws, 0)
        assert torch.equal(b.fp4q_fp8_gemm_fwd(X, W, ws=ws), want) and b.fp4q_workspace_status(ws) == 0


def test_sizes_at_which_the_plan_changes():
    # Clusters of every size, single CTAs' and pairs' tiles, with edges.
    ws = b.alloc_workspace("cuda")
    for t, n, k in ((70, 100, 2000), (129, 257, 1500), (200, 1003, 2731), (260, 900, 640), (500, 2000, 300), (1025, 1500, 260), (2100, 3000, 130)):
        check_all(t, n, k, b.OUT_F32, ws)


@pytest.mark.parametrize("dt", [b.OUT_BF16, b.OUT_F32])
@pytest.mark.parametrize("t,n,k", [(2300, 2148, 1111), (1100, 2300, 2148), (2100, 1200, 2400), (1500, 5000, 1030)])
def test_last_rounds_of_half_tiles(t, n, k, dt):
    # A few tiles of 256 x 256 more than there are pairs of CTAs; the first two with columns of which the last tile's second half has none.
    check_all(t, n, k, dt, b.alloc_workspace("cuda"))


def test_rows_behind_32_bits():
    # More than 2^31 elements between the first row of a matrix and its last: codes in a buffer of long rows, of which the product reads and the quantizer writes a few columns.
    x = randn(1, 3, 256).to(torch.bfloat16)
    far = torch.empty(3 << 30, dtype=torch.uint8, device="cuda")
    q = far.as_strided((3, 256), ((1 << 30) + (1 << 28), 1))
    t = b.fp4q_fp8_quantize(x, want_t=False)
    out = b.Fp8Tensor(3, 256, q, torch.empty(3, 2, device="cuda"))
    b.fp4q_fp8_quantize(x, out=out)
    assert torch.equal(out.q, t.q) and torch.equal(out.scale, t.scale)
    W = b.fp4q_fp8_quantize(randn(2, 300, 256), square=True)
    assert torch.equal(b.fp4q_fp8_gemm_fwd(out, W), b.fp4q_fp8_gemm_fwd(t, W))


def test_refusals():
    x = randn(1, 40, 100).to(torch.bfloat16)
    X, W = b.fp4q_fp8_quantize(x), b.fp4q_fp8_quantize(randn(2, 60, 100), square=True)
    for bad in (lambda: b.fp4q_fp8_quantize(x.half()), lambda: b.fp4q_fp8_quantize(x.T), lambda: b.fp4q_fp8_quantize(x[0]), lambda: b.fp4q_fp8_quantize(x, want=False, want_t=False),
                lambda: b.fp4q_fp8_quantize(x, out=X, square=True), lambda: b.fp4q_fp8_quantize(x, out=b.Fp8Tensor(40, 100, X.q[:, :96], X.scale)),
                lambda: b.fp4q_fp8_quantize(x[:1], out=b.Fp8Tensor(1, 100, torch.empty(1, 100, dtype=torch.uint8, device="cuda"), X.scale[:1])),   # no room behind its last element
                lambda: b.fp4q_fp8_quantize(x, out=b.Fp8Tensor(40, 100, X.q, X.scale.double())), lambda: b.fp4q_fp8_gemm_fwd(X, W, dt=7), lambda: b.fp4q_fp8_gemm_fwd(b.Fp8Tensor(40, 100, None, None), W),
                lambda: b.fp4q_fp8_gemm_fwd(X, W, out=torch.empty(40, 60, device="cuda")), lambda: b.fp4q_fp8_gemm_fwd(b.Fp8Tensor(41, 100, X.q, X.scale), W),
                lambda: b.fp4q_fp8_gemm_fwd(b.Fp8Tensor(40, 100, X.q, X.scale.view(torch.uint8)), W)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: b.fp4q_fp8_gemm_fwd(W, X), lambda: b.fp4q_fp8_gemm_fwd(X, X), lambda: b.fp4q_fp8_gemm_dgrad(X, b.Fp8Tensor(100, 60, W.q_t, W.scale.T.contiguous(), None, None, True)),
                lambda: b.fp4q_fp8_gemm_fwd(X, W, ws=torch.zeros(8, dtype=torch.uint8, device="cuda")), lambda: b.fp4q_fp8_quantize(x, out=b.Fp8Tensor(41, 100, torch.empty(41, 112, dtype=torch.uint8, device="cuda"), torch.empty(41, 1, device="cuda")))):
        with pytest.raises(b.Fp4qError):
            bad()
