"""The norm with its residual and 8-bit outputs, and its gradients, against the formulas in 64 bits.

Tolerances.  A thread adds up 16 squares a chunk (up to four) one after the other, then come at most ten steps of shuffles: their sum is off by (16 chunks + 10) 2^-24 of itself, its root by half of that, and
division, addition, root and reciprocal by 2^-24 each; y has two more roundings.  The same counts hold for the backward pass's mean.  A sum over rows has one rounding for every row that a CTA adds, for the CTAs' sums in
eights and for what joins them."""
import pytest
import torch

from paper_2607_24953_b200 import binding as b

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def chunks(cols):
    s = -(-cols // 16)
    return 1 if s <= 512 else 2 if s <= 1024 else 4


def pitched(t, ld, start=0):
    """t in rows of pitch ld that begin `start` elements into a buffer."""
    buf = torch.full((start + t.shape[0] * ld + 16,), 3.0, dtype=t.dtype, device="cuda")
    v = buf[start:].as_strided(t.shape, (ld, 1), start)
    v.copy_(t)
    return v


def mx(v):
    """(codes, scale bytes) of FP32 v by the MXFP8 rule: S the least power of two with 448 S >= M, not below 2^-127."""
    r, c = v.shape
    f = torch.nn.functional.pad(v, (0, -c % 32)).reshape(r, -1, 32).double()
    m, e = torch.frexp(f.abs().amax(2) / 448)
    e = torch.where(m == 0.5, e - 1, e)
    e = torch.where(f.abs().amax(2) > 0, e, -127).clamp_min(-127)
    q = (f * torch.exp2(-e.double())[..., None]).float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return q.reshape(r, -1), (e + 127).to(torch.uint8)


def fp8(v):
    r, c = v.shape
    f = torch.nn.functional.pad(v, (0, -c % 128)).reshape(r, -1, 128)
    m = f.abs().amax(2).clamp_min(2.0 ** -100)
    q = (f * (448.0 / m.double()).float()[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return q.reshape(r, -1)[:, :c], (m.double() / 448).float()


def check_forward(x, w, res, fmt):
    rows, cols = x.shape
    out = b.alloc_norm(x, res, y=False, q=fmt, rstd=True)
    out.y = torch.full((rows, (cols + 3) // 4 * 4 + 4), 5.0, device="cuda")[:, :cols]
    n = b.fp4q_rms_norm(x, w, res, eps=EPS, out=out)
    assert n is out
    if res is None:
        h = x
    else:
        h = (x.float() + res.float()).to(res.dtype)
        assert torch.equal(n.h, h)
    f = h.double()
    mean = (f * f).mean(1)
    r = 1 / torch.sqrt(mean + EPS)
    off = ((16 * chunks(cols) + 10) / 2 + 4) * U
    assert ((n.rstd.double() - r).abs() <= r * off).all()
    y = f * r[:, None] * (1 if w is None else w.double())
    assert ((n.y.double() - y).abs() <= y.abs() * (off + 2 * U) + 1e-45).all()
    assert (torch.as_strided(n.y, (rows, 4), (n.y.stride(0), 1), cols + (-cols) % 4) == 5).all()   # what lies behind the rows
    if fmt:
        q, s = (mx if fmt == b.Q_MXFP8 else fp8)(n.y)
        assert torch.equal(n.q[:, :q.shape[1]], q) and torch.equal(n.scale, s)
    again = b.fp4q_rms_norm(x, w, res, eps=EPS, y=True, q=fmt, rstd=True)
    assert torch.equal(again.y, n.y.to(BF16)) and torch.equal(again.rstd, n.rstd)
    if fmt:
        assert torch.equal(again.q, n.q) and torch.equal(again.scale, n.scale)


SIZES = [(1, 1), (1, 4096), (3, 16), (37, 48), (1000, 96), (5, 300), (20, 512), (9, 513), (33, 2731), (4, 8192), (3, 8200), (2, 16384), (2, 16391), (1, 65536), (5000, 40)]


@pytest.mark.parametrize("types", [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(rows, cols, types):
    x, res, w = (randn(1, rows, cols) * torch.exp(randn(2, rows, cols))).to(types[0]), randn(3, rows, cols).to(types[1]) * 3, 1 + randn(4, cols) * 0.3
    check_forward(x, w, res, b.Q_FP8)
    check_forward(x, w.to(BF16), None, b.Q_MXFP8)
    check_forward(x, None, res, b.Q_NONE)


@pytest.mark.parametrize("types", [(BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("cols,ld,start", [(40, 41, 1), (770, 777, 3), (2731, 2731, 0), (2731, 2740, 5), (600, 601, 2), (33, 35, 7)])
def test_rows_that_start_anywhere(cols, ld, start, types):
    x, res = pitched(randn(1, 50, cols).to(types[0]), ld, start), pitched(randn(2, 50, cols).to(types[1]), ld + 2, start + 1)
    w = randn(3, cols)
    check_forward(x, w, res, b.Q_FP8)
    # outputs in such rows too, nothing written beside them
    y, h = pitched(torch.zeros(50, cols, dtype=BF16, device="cuda"), ld, start), pitched(torch.zeros(50, cols, dtype=types[1], device="cuda"), ld + 3, start)
    b.fp4q_rms_norm(x, w, res, out=b.NormOut(h=h, y=y))
    want = b.fp4q_rms_norm(x, w, res)
    assert torch.equal(y, want.y) and torch.equal(h, want.h)
    for t in (y, h):
        assert t.untyped_storage().nbytes() >= (start + 50 * t.stride(0)) * t.element_size()
        flat = torch.empty(0, dtype=t.dtype, device="cuda").set_(t.untyped_storage())
        mark = torch.zeros(flat.shape, dtype=torch.bool, device="cuda")
        mark.as_strided(t.shape, t.stride(), t.storage_offset()).fill_(True)
        assert (flat[~mark] == 3).all()
    # in place
    same = res.clone() if res.is_contiguous() else pitched(res, ld + 2, start + 1)
    b.fp4q_rms_norm(x, w, same, out=b.NormOut(h=same, y=y))
    assert torch.equal(same, want.h) and torch.equal(y, want.y)


def test_zeros_infinities_and_nan_go_where_the_formulas_take_them():
    x = randn(1, 6, 300)
    x[0] = 0
    x[1, 7], x[2, 299] = float("inf"), float("nan")
    x[4] *= 1e-20
    n = b.fp4q_rms_norm(x, None, q=b.Q_FP8, rstd=True)
    assert not n.y[0].any() and not n.q[0, :300].any()
    assert n.rstd[1] == 0 and n.y[1, 7].isnan() and not n.y[1, :7].any() and not n.y[1, 8:].any()
    assert n.y[2].isnan().all() and (n.q[2, :300] == 0x7F).all() and n.q[1, 7] == 0x7F
    assert n.y[3:].isfinite().all() and n.rstd[4] == torch.tensor(1e-6).rsqrt().item() or abs(float(n.rstd[4]) - 1000) < 1e-3
    m = b.fp4q_rms_norm(x, None, q=b.Q_MXFP8)
    assert not m.q[2].any() and (m.scale[2] == 0).all()      # as the MXFP8 quantizers: NaN becomes 0
    clean = x.clone()
    clean[1:3] = 1
    assert torch.equal(b.fp4q_rms_norm(clean, None).y[3:], n.y[3:])   # other rows are untouched by it


def check_backward(dy, h, w, dh, want_dw=True):
    rows, cols = h.shape
    rstd = torch.rsqrt(h.double().square().mean(1) + EPS).float()
    dx, dw = b.fp4q_rms_norm_bwd(dy, h, rstd, w, dh=dh, want_dweight=want_dw)
    d, f, r = dy.double(), h.double(), rstd.double()[:, None]
    g = d if w is None else d * w.double()
    x = f * r
    mean, size = (g * x).mean(1, keepdim=True), (g * x).abs().mean(1, keepdim=True)
    want = r * (g - x * mean) + (0 if dh is None else dh.double())
    k = 16 * chunks(cols) + 10 + 4                                  # roundings of the mean
    tol = r * (g.abs() * 4 * U + x.abs() * size * (k + 4) * U) + want.abs() * half_step(h.dtype) * (1 + 2.0 ** -7) + (0 if dh is None else dh.double().abs() * U) + 1e-45
    # where the result cancels, FP32 roundings of its terms remain
    tol = tol + (r * (g.abs() + x.abs() * mean.abs()) + (0 if dh is None else dh.double().abs())) * 2 * U
    assert dx.dtype == h.dtype and ((dx.double() - want).abs() <= tol).all(), float(((dx.double() - want).abs() / tol).max())
    if not want_dw:
        assert dw is None
        return
    sums = (d * x).sum(0)
    k = rows / 8 + 296 / 8 + 300 if rows > 296 else 8 + 40
    assert ((dw.double() - sums).abs() <= (d * x).abs().sum(0) * k * U + 1e-45).all()
    before = randn(9, cols)
    acc = before.clone()
    b.fp4q_rms_norm_bwd(dy, h, rstd, w, dh=dh, dweight=acc, accumulate=True)
    assert torch.equal(acc, before + dw)
    none, _ = b.fp4q_rms_norm_bwd(dy, h, rstd, w, dh=dh, want_dweight=False)
    assert torch.equal(none, dx)


@pytest.mark.parametrize("types", [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("rows,cols", SIZES + [(1999, 731), (700, 9000), (3000, 4096)])
def test_backward(rows, cols, types):
    dy, h, dh = (randn(1, rows, cols) * torch.exp(2 * randn(2, rows, 1))).to(types[0]), randn(3, rows, cols).to(types[1]) * 2, randn(4, rows, cols).to(types[1])
    check_backward(dy, h, 1 + 0.3 * randn(5, cols), dh)
    check_backward(dy, h, (1 + 0.3 * randn(5, cols)).to(BF16), None)
    check_backward(dy, h, None, dh)


@pytest.mark.parametrize("cols,ld,start", [(40, 41, 1), (770, 777, 3), (2731, 2731, 0), (601, 640, 5)])
def test_backward_of_rows_that_start_anywhere_and_in_place(cols, ld, start):
    for ty, th in ((BF16, BF16), (F32, BF16), (BF16, F32)):
        dy, h, dh = pitched(randn(1, 60, cols).to(ty), ld, start), pitched(randn(2, 60, cols).to(th), ld + 1, start + 2), pitched(randn(3, 60, cols).to(th), ld + 3, start)
        w = randn(4, cols)
        check_backward(dy, h, w, dh)
        rstd = torch.ones(60, device="cuda")
        want, dw = b.fp4q_rms_norm_bwd(dy, h, rstd, w, dh=dh)
        got, dw2 = b.fp4q_rms_norm_bwd(dy, h, rstd, w, dh=dh, out=dh)
        assert got is dh and torch.equal(dh, want) and torch.equal(dw, dw2)


def test_no_rows():
    h = torch.empty(0, 40, device="cuda")
    dw = torch.ones(40, device="cuda")
    b.fp4q_rms_norm_bwd(h, h, torch.empty(0, device="cuda"), None, dweight=dw, accumulate=True)
    assert (dw == 1).all()
    b.fp4q_rms_norm_bwd(h, h, torch.empty(0, device="cuda"), None, dweight=dw)
    assert not dw.any()
    assert b.fp4q_rms_norm(h, None, q=b.Q_FP8, rstd=True).y.shape == (0, 40)


def test_gradients_against_differences():
    # Central differences of the formula in 64 bits along random directions: off by the step's square, and by the kernel's FP32 roundings, both far below 1e-4.
    rows, cols, step = 20, 200, 1e-4
    h, w, dy = randn(1, rows, cols), 1 + 0.3 * randn(2, cols), randn(3, rows, cols)

    def loss(h, w):
        return (h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * w * dy.double()).sum()
    rstd = b.fp4q_rms_norm(h, w, rstd=True).rstd
    dx, dw = b.fp4q_rms_norm_bwd(dy, h, rstd, w)
    for seed in range(4):
        v, u = randn(10 + seed, rows, cols).double(), randn(20 + seed, cols).double()
        slope = (loss(h.double() + step * v, w.double() + step * u) - loss(h.double() - step * v, w.double() - step * u)) / (2 * step)
        got = (dx.double() * v).sum() + (dw.double() * u).sum()
        assert abs(float(slope - got)) <= 1e-4 * float((dx.double() * v).abs().sum() + (dw.double() * u).abs().sum())


def test_refusals():
    x, w = randn(1, 8, 64).to(BF16), randn(2, 64)
    rstd = torch.ones(8, device="cuda")
    for bad in (lambda: b.fp4q_rms_norm(x.half()), lambda: b.fp4q_rms_norm(x.T), lambda: b.fp4q_rms_norm(x[0]), lambda: b.fp4q_rms_norm(x, w[:63]), lambda: b.fp4q_rms_norm(x, w.double()),
                lambda: b.fp4q_rms_norm(x, w, x[:4]), lambda: b.fp4q_rms_norm(x, w, x.cpu()), lambda: b.fp4q_rms_norm(x, q=5), lambda: b.fp4q_rms_norm(x, w, x, out=b.NormOut(y=x.clone())),
                lambda: b.fp4q_rms_norm(x, w, x, out=b.NormOut(h=x.float())), lambda: b.fp4q_rms_norm(x, out=b.NormOut(q=torch.empty(8, 64, dtype=torch.uint8, device="cuda"))),
                lambda: b.fp4q_rms_norm(x, out=b.NormOut(rstd=rstd[:7])), lambda: b.fp4q_rms_norm(x, out=b.NormOut(y=x[:, :63])),
                lambda: b.fp4q_rms_norm_bwd(x[:4], x, rstd), lambda: b.fp4q_rms_norm_bwd(x, x, rstd[:3]), lambda: b.fp4q_rms_norm_bwd(x, x, rstd, w, dh=x.float()),
                lambda: b.fp4q_rms_norm_bwd(x, x, rstd, w, out=x.float()), lambda: b.fp4q_rms_norm_bwd(x, x, rstd, w, dweight=w[:5])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: b.fp4q_rms_norm(x, eps=-1.0), lambda: b.fp4q_rms_norm(torch.empty(1, 65537, device="cuda")), lambda: b.fp4q_rms_norm_bwd(x, x, rstd, w, scratch=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(b.Fp4qError):
            bad()


def test_rows_behind_32_bits():
    far = torch.empty(3 << 30, dtype=BF16, device="cuda")
    x = far.as_strided((3, 400), ((1 << 30) + (1 << 28) + 1, 1))
    x.copy_(randn(1, 3, 400))
    near, w = x.clone(), randn(2, 400)
    a, c = b.fp4q_rms_norm(x, w, q=b.Q_FP8, rstd=True), b.fp4q_rms_norm(near, w, q=b.Q_FP8, rstd=True)
    assert torch.equal(a.y, c.y) and torch.equal(a.q[:, :400], c.q[:, :400])
    dx = b.fp4q_rms_norm_bwd(near, x, a.rstd, w, out=x)[0]
    assert torch.equal(dx, b.fp4q_rms_norm_bwd(near, near, a.rstd, w)[0])
