"""The norm of many gradients and their clipping, against 64 bits.  The norm: runs of 32 squares in FP32 are off by 32 * 2^-24 of themselves, the root by half of that, and it is rounded once; a clipped
element by the roundings of the factor (norm + eps, the quotient) and its own."""
import math

import pytest
import torch

from paper_2607_24953_b200 import autograd, binding as b

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def true_norm(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


def check(ts, max_norm, outs=None, eps=1e-6):
    before, true = [t.clone() for t in ts], true_norm(ts)
    norm = b.fp4q_clip_grad_norm(ts, max_norm, outs=outs, eps=eps)
    assert norm.shape == () and abs(float(norm) - true) <= true * 18 * U
    c = min(1.0, max_norm / (true + eps))
    for t, o, was in zip(ts, outs or ts, before):
        if outs is not None:
            assert torch.equal(t, was)
        want = was.double() * c
        if c == 1.0:
            assert torch.equal(o, was.to(o.dtype))
        assert ((o.double() - want).abs() <= want.abs() * (torch.finfo(o.dtype).eps / 2 + 22 * U) * (1 + 2.0 ** -6) + 2.0 ** -149).all()
    return norm


SHAPES = [(1,), (7,), (8,), (256, 256), (3, 5), (1000, 33), (2048,), (0, 5), (4, 4, 4), (1, 8193), (300, 777)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("out", [None, BF16, F32])
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_tensors_of_all_sizes(dtype, out, max_norm):
    ts = [randn(i, *s).to(dtype) for i, s in enumerate(SHAPES)]
    check(ts, max_norm, None if out is None else [torch.empty(t.shape, dtype=out, device="cuda") for t in ts])


def test_types_side_by_side_and_many_tensors():
    for count in (1, 2, 56, 57, 450, 451, 1000):
        ts = [randn(i, 1 + i % 300).to(BF16 if i % 3 else F32) for i in range(count)]
        check(ts, 1.0)
        check([torch.zeros(0, device="cuda")] + ts, 1.0, [torch.empty(0, device="cuda")] + [torch.empty(t.shape, device="cuda") for t in ts])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_alignments(dtype):
    flat = randn(1, 100000).to(dtype)
    views = [flat[1:1000], flat[1003:2002], flat[2002:2003], flat[3000:3000 + 70 * 41].view(70, 41)[:, :33], flat[10001:10001 + 30 * 64].view(30, 64)[:, 3:60],
             flat[20000:20000 + 600].view(20, 30).T, flat[30001:30001 + 4 * 6 * 16].view(4, 6, 16)[:, :, :9], flat[40005:40005 + 300 * 9].view(300, 9)[:, :2], flat[50000:51000].view(1, 1000)[:, 2:900]]
    keep = flat.clone()
    mark = torch.zeros(flat.shape, dtype=torch.bool, device="cuda")
    for v in views:
        mark.as_strided(v.shape, v.stride(), v.storage_offset()).fill_(True)
    check(views, 0.25)
    assert torch.equal(flat[~mark], keep[~mark]) and not torch.equal(flat[mark], keep[mark])
    for out in (BF16, F32):                                     # into entries of other strides
        outs = [torch.empty(v.shape, dtype=out, device="cuda") for v in views]
        outs[5] = torch.empty(20, 30, dtype=out, device="cuda").T
        check(views, 0.1, outs)
    shifted = [torch.empty(v.numel() + 1, dtype=dtype, device="cuda")[1:].view(v.shape) for v in views[:2]]
    check(views[:2], 0.05, shifted)


def test_single_elements_of_any_strides():
    flat = randn(1, 64)
    one, row = flat[::8][:1], flat.view(8, 8)[:1]
    check([one, row], 0.1, [torch.empty(1, device="cuda"), torch.empty(1, 8, device="cuda")])


def test_numbers_whose_squares_leave_fp32():
    for scale in (1e-30, 1e-22, 1e25, 3e37):
        ts = [randn(1, 5000) * scale, randn(2, 3) * scale]
        norm = b.fp4q_global_norm(ts)
        true = true_norm(ts)
        assert abs(float(norm) - true) <= true * 18 * U if true < 3.4e38 else math.isinf(float(norm))
    ts = [randn(1, 5000) * 1e-30, randn(2, 5000)]
    assert abs(float(b.fp4q_global_norm(ts)) - true_norm(ts)) <= true_norm(ts) * 18 * U
    assert float(b.fp4q_global_norm([torch.zeros(100, device="cuda")])) == 0.0
    assert float(b.fp4q_global_norm([torch.empty(0, 3, device="cuda")])) == 0.0


def test_infinities_and_nan():
    g = [randn(1, 100), randn(2, 3000)]
    g[1][5] = float("nan")
    assert b.fp4q_clip_grad_norm(g, 1.0).isnan() and all(t.isnan().all() for t in g)
    g = [randn(1, 100), randn(2, 3000)]
    g[1][5] = float("inf")
    assert b.fp4q_clip_grad_norm(g, 1.0).isinf() and not g[0].any() and g[1][5].isnan() and not g[1][6:].any()


def test_zeros_stay_zeros_and_a_zero_bound():
    g = [torch.zeros(50, device="cuda")]
    assert float(b.fp4q_clip_grad_norm(g, 1.0)) == 0 and not g[0].any()
    g = [randn(1, 50)]
    b.fp4q_clip_grad_norm(g, 0.0)
    assert not g[0].any()


def test_a_norm_from_elsewhere():
    g = [randn(1, 500), randn(2, 500).to(BF16)]
    want = [(t.double() * 0.25).to(t.dtype) for t in g]
    norm = torch.tensor(4.0, device="cuda")
    assert b.fp4q_clip_by_norm(g, norm, 1.0, eps=0.0) is g
    assert all(torch.equal(p, q) for p, q in zip(g, want))     # a power of two: exact


def test_the_order_is_fixed():
    ts = [randn(i, 1000 + 977 * i) for i in range(30)]
    first = b.fp4q_global_norm(ts)
    assert all(torch.equal(first, b.fp4q_global_norm(ts)) for _ in range(5))


def test_parameters_gradients():
    ps = [torch.nn.Parameter(randn(i, 30, 20)) for i in range(4)]
    for p in ps[:3]:
        p.grad = randn(9, 30, 20) * 5
    true = true_norm([p.grad for p in ps[:3]])
    norm = autograd.clip_grad_norm_(ps, 1.0)
    assert abs(float(norm) - true) <= true * 18 * U and abs(true_norm([p.grad for p in ps[:3]]) - 1) < 1e-5
    assert float(autograd.clip_grad_norm_([ps[3]], 1.0)) == 0
    assert float(autograd.clip_grad_norm_(ps[0], 10.0)) < 1


def test_refusals():
    g = [randn(1, 10)]
    for bad in ([randn(1, 10).double()], [torch.zeros(10)], [], [g[0], torch.zeros(3)], [randn(1, 10, 10)[:, ::2]], [g[0].expand(3, 10)]):
        with pytest.raises(ValueError):
            b.fp4q_global_norm(bad)
    with pytest.raises(ValueError, match="twice"):
        b.fp4q_clip_grad_norm([g[0], g[0]], 1.0)
    for outs in ([], [randn(1, 9)], [randn(1, 10).half()], [torch.zeros(10)]):
        with pytest.raises(ValueError):
            b.fp4q_clip_grad_norm(g, 1.0, outs=outs)
    for max_norm, eps in ((-1.0, 1e-6), (float("nan"), 1e-6), (1.0, -1.0)):
        with pytest.raises(b.Fp4qError):
            b.fp4q_clip_grad_norm(g, max_norm, eps=eps)
    with pytest.raises(b.Fp4qError):
        b.fp4q_global_norm(g, scratch=torch.empty(8, dtype=torch.uint8, device="cuda"))
