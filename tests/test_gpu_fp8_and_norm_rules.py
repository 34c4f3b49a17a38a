"""The 8-bit formats' rules seen from other sides: the norm's MXFP8 output against the quantizer of that format and through its product, how near codes are to what they stand for, the
same call twice and from two threads, rows beside rows of infinities, gradients of more than 2^32 bytes."""
import threading

import pytest
import torch

from paper_2607_24953_b200 import binding as b

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 4096), (37, 64), (300, 1000), (9, 33), (5, 8200)])
def test_the_norms_mxfp8_output_is_the_quantizers(rows, cols, dtype):
    # Signs alone have a mean square of 1 (at these widths 1 / cols in FP32 times cols is 1), so that the norm's output is the weight with these signs, BF16 numbers, which the quantizer reads as they are.
    x = torch.where(randn(1, rows, cols) < 0, -1.0, 1.0)
    w = (randn(2, cols) * torch.exp(3 * randn(3, cols))).to(BF16)
    n = b.fp4q_rms_norm(x.to(dtype), w, eps=0.0, q=b.Q_MXFP8, rstd=True)
    assert (n.rstd == 1).all() and torch.equal(n.y, x.to(BF16) * w)
    q, s = b.fp4q_mxfp8_quantize1d(n.y)
    assert torch.equal(n.scale[:, :s.shape[1]], s) and torch.equal(n.q[:, :cols], q[:, :cols])


@pytest.mark.parametrize("T,K,N", [(1, 4096, 256), (200, 512, 128), (77, 1000, 96)])
def test_the_norms_mxfp8_output_goes_into_its_product(T, K, N):
    x, w = randn(1, T, K).to(BF16), 1 + 0.3 * randn(2, K)
    n = b.fp4q_rms_norm(x, w, q=b.Q_MXFP8)
    (wq, ws), (vq, vs) = (b.fp4q_mxfp8_quantize1d((randn(i, N, K) * 0.05).to(BF16)) for i in (3, 4))
    got = b.fp4q_mxfp8_qk(n.q, n.scale, wq, ws, vq, vs, T, K, N, dt=b.OUT_F32)
    values = lambda q, s: q[:, :K].view(torch.float8_e4m3fn).double() * torch.exp2(s.double() - 127).repeat_interleave(32, 1)[:, :K]  # noqa: E731
    X = values(n.q, n.scale)
    for y, (q, s) in zip(got, ((wq, ws), (vq, vs))):
        W = values(q, s)
        want, size = X @ W.T, X.abs() @ W.abs().T
        # the tensor cores' sums of 32 products cut off at 2^-22 of the largest term at worst, K / 32 of them one after the other
        assert ((y.double() - want).abs() <= size * (K / 32 + 2) * 2.0 ** -22).all()
    # and it is the norm: an element is off by half a step, 2^-4 of itself or 2^-10 of its scale, and by FP32's roundings
    f = x.double()
    want = f * torch.rsqrt((f * f).mean(1, keepdim=True) + 1e-6) * w.double()
    step = torch.exp2(n.scale.double() - 127).repeat_interleave(32, 1)[:, :K] * 2.0 ** -10
    assert ((X - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, step) * (1 + 2.0 ** -10)).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("square", [False, True])
def test_codes_are_the_nearest_ones_and_the_same_every_time(square, dtype):
    # The rule multiplies by 448 / M and the scale is M / 448, both rounded: a code is the nearest to x / scale but for quotients within 3 * 2^-24 of a border, where either is as near.
    x = (randn(1, 700, 1000) * torch.exp(1.5 * randn(2, 700, 1)) * 1e-3).to(dtype)
    t = b.fp4q_fp8_quantize(x, square=square)
    for q, scale, m in ((t.q[:, :1000], t.scale, x), (t.q_t[:, :700], t.scale.T if square else t.scale_t, x.T)):
        s = scale.double().repeat_interleave(128, 0)[:m.shape[0]] if square else scale.double()
        v = m.double() / s.repeat_interleave(128, 1)[:, :m.shape[1]]
        c = q.view(torch.float8_e4m3fn).double()
        ulp = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)      # of E4M3 at the quotient
        assert ((c - v).abs() <= ulp / 2 + v.abs() * 3 * 2.0 ** -24).all()
    for _ in range(5):
        again = b.fp4q_fp8_quantize(x, square=square)
        assert torch.equal(again.q[:, :1000], t.q[:, :1000]) and torch.equal(again.q_t[:, :700], t.q_t[:, :700]) and torch.equal(again.scale, t.scale)


def test_rows_beside_infinities_and_nan_are_what_they_are_without():
    x = randn(1, 6, 300)
    x[0], x[1, 7], x[2, 299] = 0, float("inf"), float("nan")
    x[4] *= 1e-20
    n = b.fp4q_rms_norm(x, None, q=b.Q_FP8, rstd=True)
    assert n.y[3:].isfinite().all()
    assert abs(float(n.rstd[4]) - 1000) < 1e-3
    alone = b.fp4q_rms_norm(x[3:].contiguous(), None, q=b.Q_FP8, rstd=True)
    assert torch.equal(n.y[3:], alone.y) and torch.equal(n.q[3:], alone.q) and torch.equal(n.scale[3:], alone.scale) and torch.equal(n.rstd[3:], alone.rstd)


def test_from_two_threads():
    def work(seed):
        x, w = randn(seed, 300, 520).to(BF16), randn(seed + 1, 260, 520) * 0.05
        g = 1 + 0.2 * randn(seed + 2, 520)
        dy = randn(seed + 3, 300, 260).to(BF16)

        def step(ws):
            n = b.fp4q_rms_norm(x, g, x, q=b.Q_FP8, rstd=True)
            W, D = b.fp4q_fp8_quantize(w, square=True), b.fp4q_fp8_quantize(dy)
            y = b.fp4q_fp8_gemm_fwd(b.Fp8Tensor(300, 520, n.q, n.scale), W, ws=ws)
            dx, dg = b.fp4q_rms_norm_bwd(b.fp4q_fp8_gemm_dgrad(D, W, ws=ws), n.h, n.rstd, g)
            dw = b.fp4q_fp8_gemm_wgrad(D, b.fp4q_fp8_quantize(n.y, want=False), ws=ws)
            norm = b.fp4q_clip_grad_norm([dw, dg], 0.1)
            return [y, dx, dg, dw, norm]
        return step
    steps = [work(100 * i) for i in range(2)]
    want = [s(b.alloc_workspace("cuda")) for s in steps]
    torch.cuda.synchronize()
    got, failed = [[], []], []

    def thread(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                ws = b.alloc_workspace("cuda")
                for _ in range(30):
                    got[i].append(steps[i](ws))
                torch.cuda.current_stream().synchronize()
        except BaseException as e:  # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=thread, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    for i in range(2):
        for out in got[i]:
            assert all(torch.equal(p, q) for p, q in zip(out, want[i]))


@pytest.mark.parametrize("shape,pitch", [((2500, 1 << 20), None), ((3, 1 << 20), (1 << 30) + 8)])
def test_gradients_of_more_than_32_bits_of_bytes(shape, pitch):
    if pitch is None:
        g = torch.empty(shape, dtype=BF16, device="cuda")
        for rows in g.split(100):
            rows.copy_(randn(int(rows.data_ptr() % 1000), 1, shape[1]).expand_as(rows))
    else:
        g = torch.empty(3 * pitch, dtype=BF16, device="cuda").as_strided(shape, (pitch, 1))
        g.copy_(randn(1, *shape))
    total = sum(float(rows.double().square().sum()) for rows in g.split(50))
    first, last = g[:1].clone(), g[-1:].clone()
    norm = b.fp4q_clip_grad_norm([g], 1.0)
    assert abs(float(norm) - total ** 0.5) <= total ** 0.5 * 18 * 2.0 ** -24
    c = 1.0 / (total ** 0.5 + 1e-6)
    for now, was in ((g[:1], first), (g[-1:], last)):
        want = was.double() * c
        assert ((now.double() - want).abs() <= want.abs() * (2.0 ** -8 + 22 * 2.0 ** -24) * (1 + 2.0 ** -6) + 2.0 ** -134).all()
