"""BF16 products of groups that start anywhere, against 64-bit products of the same operands.

Tolerance, per element.  With S = sum |a||b|: an accumulator takes 16 products at a time; the sum of it and the products is cut off to FP32 below
2^-23 of its largest term, and so may each product be before it is added, together less than 2^-22 S for one instruction.  BF16 outputs
take ceil(K/16) instructions and one rounding, 2^-8 of the value.  FP32 outputs take at most 32 instructions per partial sum and
ceil(K/512) roundings to nearest, 2^-24 S each, and one when something is added to."""
import math

import numpy as np
import pytest
import torch

from paper_2607_24953_b200 import autograd, binding as b

pytestmark = pytest.mark.gpu


def rows16(t, extra=0):
    """t in rows of whole 16 bytes (and `extra` times 16 bytes more), NaN in what does not belong to it."""
    buf = torch.full((t.shape[0], (t.shape[1] + 7) // 8 * 8 + 8 * extra), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def offsets(values):
    return torch.tensor(values, dtype=torch.int64, device="cuda")


def groups(values, T):
    v = [max(0, min(T, x)) for x in values]
    for i in range(1, len(v)):
        v[i] = max(v[i], v[i - 1])
    return list(zip(v[:-1], v[1:]))


def reference(op, a, w, spans):
    """The product and its S, in 64 bits; rows of nobody are NaN."""
    a, w = a.double(), w.double()
    if op == "wgrad":
        y = torch.cat([a[i:j].T @ w[i:j] for i, j in spans])
        return y, torch.cat([a[i:j].abs().T @ w[i:j].abs() for i, j in spans])
    n = w.shape[0] // len(spans)
    y = torch.full((a.shape[0], n if op == "fwd" else w.shape[1]), float("nan"), dtype=torch.float64, device="cuda")
    s = y.clone()
    for g, (i, j) in enumerate(spans):
        m = w[g * n:(g + 1) * n]
        m = m.T if op == "fwd" else m
        y[i:j], s[i:j] = a[i:j] @ m, a[i:j].abs() @ m.abs()
    return y, s


def bound(y, s, k, dt, adds=False):
    if dt == b.OUT_BF16:
        return y.abs() * 2 ** -8 + s * math.ceil(k / 16) * 2 ** -22 + 1e-30
    return s * (min(32, math.ceil(k / 16)) * 2 ** -22 + (math.ceil(k / 512) + adds) * 2 ** -24) + y.abs() * 2 ** -24 + 1e-30


def call(op, a, w, offs, out=None, dt=b.OUT_BF16, **kw):
    f = {"fwd": b.fp4q_ragged_gemm_fwd, "dgrad": b.fp4q_ragged_gemm_dgrad, "wgrad": b.fp4q_ragged_gemm_wgrad}[op]
    return f(a, w, offs, out=out, dt=dt, **kw)


def operands(op, T, n, k, e, seed=0, extra=0):
    x, dy, w = rows16(randn(seed, T, k), extra), rows16(randn(seed + 1, T, n) * 0.1, extra), rows16(randn(seed + 2, e * n, k) * 0.05, extra)
    return {"fwd": (x, w), "dgrad": (dy, w), "wgrad": (dy, x)}[op]


CASES = [   # T, N, K, offsets
    (1, 16, 16, [0, 1]),
    (7, 8, 24, [0, 0, 3, 3, 7, 7]),
    (130, 130, 200, [0, 129, 130]),
    (300, 257, 129, [3, 3, 70, 71, 199, 288]),
    (257, 1, 1, [0, 100, 257]),
    (1000, 72, 1000, [0, 63, 127, 192, 256, 512, 1000]),
    (513, 300, 1, [0, 513]),
    (600, 520, 700, [0, 17, 17, 255, 600]),
    (5000, 264, 136, [0, 2500, 2501, 5000]),
    (40, 700, 520, list(range(41))),
]


@pytest.mark.parametrize("dt", [b.OUT_BF16, b.OUT_F32])
@pytest.mark.parametrize("op", ["fwd", "dgrad", "wgrad"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_matches_64_bit_products(case, op, dt):
    T, n, k, values = CASES[case]
    spans = groups(values, T)
    a, w = operands(op, T, n, k, len(spans), 10 * case, extra=case % 2)
    for i, j in [(0, spans[0][0]), (spans[-1][1], T)]:     # nobody's rows: what lies there must not matter
        a[i:j] = float("inf")
        if op == "wgrad":
            w[i:j] = float("nan")
    ws = b.alloc_workspace("cuda")
    rows, cols = {"fwd": (T, n), "dgrad": (T, k), "wgrad": (len(spans) * n, k)}[op]
    ld = (cols + 7) // 8 * 8 + 8
    buf = torch.full((rows + 2, ld), 7.0, dtype=torch.bfloat16 if dt == b.OUT_BF16 else torch.float32, device="cuda")
    out = buf[1:-1, :cols]
    assert call(op, a, w, offsets(values), out, dt, ws=ws) is out
    torch.cuda.synchronize()
    assert b.fp4q_workspace_status(ws) == 0
    y, s = reference(op, a, w, spans)
    length = {"fwd": k, "dgrad": n, "wgrad": max(j - i for i, j in spans)}[op]
    mine = torch.ones(rows, dtype=torch.bool, device="cuda")
    if op != "wgrad":
        mine[:spans[0][0]] = False
        mine[spans[-1][1]:] = False
    got = out.double()
    assert ((got - y).abs()[mine] <= bound(y, s, length, dt)[mine]).all()
    assert (got[~mine] == 7).all()                          # nobody's rows as they were
    assert (buf[0] == 7).all() and (buf[-1] == 7).all() and (buf[:, cols:] == 7).all()
    fresh = call(op, a, w, offsets(values), None, dt, ws=ws)
    assert torch.equal(fresh[mine], out[mine]) and not fresh[~mine].any()
    assert torch.equal(call(op, a, w, offsets(values), None, dt, ws=ws), fresh)


@pytest.mark.parametrize("op", ["fwd", "dgrad", "wgrad"])
@pytest.mark.parametrize("T,n,k,e", [(30000, 512, 264, 5), (3000, 768, 1024, 64), (64, 768, 2048, 128), (9000, 300, 1500, 20)])
def test_larger_ones_with_skewed_groups(op, T, n, k, e):
    p = np.arange(1, e + 1) ** -1.2
    counts = np.random.RandomState(e).multinomial(T - 5, p / p.sum())
    values = (5 + np.concatenate([[0], np.cumsum(counts)])).tolist()
    a, w = operands(op, T, n, k, e, e)
    y, s = reference(op, a, w, groups(values, T))
    length = {"fwd": k, "dgrad": n, "wgrad": max(counts)}[op]
    for dt in (b.OUT_BF16, b.OUT_F32):
        got = call(op, a, w, offsets(values), None, dt).double()
        rows = slice(0, None) if op == "wgrad" else slice(5, T)
        assert ((got - y).abs() <= bound(y, s, length, dt))[rows].all()
        if dt == b.OUT_F32:    # a sum of one sign, where the cut-off towards zero would add up: 512 elements' worth of it at most
            z = call(op, rows16(a.abs()), rows16(w.abs()), offsets(values), None, dt).double()
            assert ((z - s).abs() <= bound(s, s, length, dt))[rows].all()


@pytest.mark.parametrize("T,n,k,values", [(20000, 200, 300, [0, 20000]), (20000, 100, 72, [0, 7, 15000, 15001, 20000]), (9000, 512, 256, [100, 5000, 9000]),
                                          (60000, 300, 130, [0, 59000, 59900, 60000]), (3000, 64, 64, [0, 3000])])
def test_long_contractions_in_parts(T, n, k, values):
    dy, x = operands("wgrad", T, n, k, len(values) - 1)
    y, s = reference("wgrad", dy, x, groups(values, T))
    length = max(j - i for i, j in groups(values, T))
    scratch = b.alloc_ragged_wgrad_scratch(T, n, k, len(values) - 1, "cuda")
    assert scratch.numel() > 0
    for dt in (b.OUT_F32, b.OUT_BF16):
        scratch.fill_(255)                                  # any contents
        want = call("wgrad", dy, x, offsets(values), dt=dt, scratch=scratch)
        assert ((want.double() - y).abs() <= bound(y, s, length, dt)).all()
        for _ in range(3):                                  # which part comes last changes nothing
            assert torch.equal(call("wgrad", dy, x, offsets(values), dt=dt, scratch=scratch), want)
        assert torch.equal(call("wgrad", dy, x, offsets(values), dt=dt), want)
    out = randn(3, y.shape[0], (k + 3) // 4 * 4 + 4)[:, :k]
    before = out.clone()
    call("wgrad", dy, x, offsets(values), out, b.OUT_F32, accumulate=True, scratch=scratch)
    assert ((out.double() - before.double() - y).abs() <= bound(y + before.double(), s + before.double().abs(), length, b.OUT_F32, adds=True)).all()
    with pytest.raises(b.Fp4qError) as err:
        call("wgrad", dy, x, offsets(values), dt=b.OUT_F32, scratch=scratch[:256])
    assert err.value.status == 5


@pytest.mark.parametrize("T,n,k,values", [(16000, 1024, 1000, [0, 16000]), (20000, 600, 1500, [0, 300, 20000]), (40000, 520, 264, [0, 9000, 9000, 21000, 40000])])
def test_parts_of_larger_tiles_and_of_few_groups(T, n, k, values):
    dy, x = operands("wgrad", T, n, k, len(values) - 1)
    y, s = reference("wgrad", dy, x, groups(values, T))
    length = max(j - i for i, j in groups(values, T))
    scratch = b.alloc_ragged_wgrad_scratch(T, n, k, len(values) - 1, "cuda")
    assert scratch.numel() > 0
    for dt in (b.OUT_F32, b.OUT_BF16):
        scratch.fill_(255)
        want = call("wgrad", dy, x, offsets(values), dt=dt, scratch=scratch)
        assert ((want.double() - y).abs() <= bound(y, s, length, dt)).all()
        assert torch.equal(call("wgrad", dy, x, offsets(values), dt=dt, scratch=scratch), want)


@pytest.mark.parametrize("T,values", [(64, [0, 64]), (600, [0, 150, 300, 450, 600]), (200, [0] + [2 * i for i in range(1, 101)])])
def test_every_shape_of_tile(T, values):
    # few rows of one group, some of a few, two each of a hundred
    for op in ("fwd", "dgrad"):
        x, w = operands(op, T, 1000, 520, len(values) - 1)
        y, s = reference(op, x, w, groups(values, T))
        for dt in (b.OUT_BF16, b.OUT_F32):
            got = call(op, x, w, offsets(values), dt=dt)
            assert ((got.double() - y).abs() <= bound(y, s, 520 if op == "fwd" else 1000, dt)).all()


def test_no_groups_at_all_and_one_for_everything():
    a, w = operands("fwd", 300, 96, 200, 1)
    assert torch.equal(call("fwd", a, w, None), call("fwd", a, w, offsets([0, 300])))
    assert torch.equal(call("wgrad", a, a, None, dt=b.OUT_F32), call("wgrad", a, a, offsets([0, 300]), dt=b.OUT_F32))
    z = call("wgrad", a, a, offsets([5, 5, 5]))
    assert z.shape == (400, 200) and not z.any()
    z = call("fwd", a, rows16(torch.zeros(192, 200)), offsets([300, 300, 300]))
    assert z.shape == (300, 96) and not z.any()


@pytest.mark.parametrize("T,n,k", [(0, 40, 64), (30, 0, 64), (30, 40, 0)])
def test_sizes_of_zero(T, n, k):
    x, dy, w = (rows16(torch.ones(*s, device="cuda")) for s in ((T, k), (T, n), (2 * n, k)))
    offs = offsets([0, T // 2, T])
    assert call("fwd", x, w, offs).shape == (T, n) and not call("fwd", x, w, offs, dt=b.OUT_F32).any()
    dx = call("dgrad", dy, w, offs)
    assert dx.shape == (T, k) and not dx.any()
    dw = call("wgrad", dy, x, offs, dt=b.OUT_F32)
    assert dw.shape == (2 * n, k) and not dw.any()
    kept = torch.full((2 * n, max(k, 4)), 3.0, device="cuda")[:, :k]
    if T == 0:
        call("wgrad", dy, x, offs, kept, b.OUT_F32, accumulate=True)
        assert (kept == 3).all()


@pytest.mark.parametrize("T,e", [(700, 3), (9, 4), (5000, 2)])
def test_accumulation(T, e):
    values = [0] + [T * (i + 1) // e for i in range(e)]
    values[1] = 0                                           # an empty group: its part stays
    dy, x = operands("wgrad", T, 100, 136, e)
    out = randn(9, e * 100, 136)
    before = out.clone()
    call("wgrad", dy, x, offsets(values), out, b.OUT_F32, accumulate=True)
    y, s = reference("wgrad", dy, x, groups(values, T))
    assert torch.equal(out[:100], before[:100])
    assert ((out.double() - before.double() - y).abs() <= bound(y + before.double(), s + before.double().abs(), T, b.OUT_F32, adds=True)).all()
    with pytest.raises(b.Fp4qError):
        call("wgrad", dy, x, offsets(values), out.to(torch.bfloat16), b.OUT_BF16, accumulate=True)


@pytest.mark.parametrize("op", ["fwd", "dgrad", "wgrad"])
def test_a_group_does_not_see_its_neighbours(op):
    T, n, k, values = 400, 136, 200, [0, 101, 130, 131, 260, 400]
    a, w = operands(op, T, n, k, 5)
    want = call(op, a, w, offsets(values), dt=b.OUT_F32)
    for bad in (float("nan"), float("inf")):
        a2, w2 = a.clone(), w.clone()
        a2[101:130] = bad
        a2[131:260] = bad
        if op == "wgrad":
            w2[101:130] = bad
            w2[131:260] = bad
        got = call(op, rows16(a2), rows16(w2), offsets(values), dt=b.OUT_F32)
        keep = [slice(0, 101), slice(130, 131), slice(260, 400)] if op != "wgrad" else [slice(g * n, g * n + n) for g in (0, 2, 4)]
        for rows in keep:
            assert torch.equal(got[rows], want[rows])


@pytest.mark.parametrize("values", [[0, 900, 20, 300], [-50, 10, 10, 10 ** 12], [200, 100, 50, 0], [0, 2 ** 40, -2 ** 40, 300]])
def test_offsets_that_are_no_boundaries_touch_nothing_else(values):
    T, n, k = 300, 64, 72
    spans = groups(values, T)
    for op in ("fwd", "dgrad", "wgrad"):
        a, w = operands(op, T, n, k, 3)
        got = call(op, a, w, offsets(values), dt=b.OUT_F32).double()
        y, s = reference(op, a, w, spans)
        y, s = y.nan_to_num(0.0), s.nan_to_num(0.0)
        assert ((got - y).abs() <= bound(y, s, 512, b.OUT_F32)).all()


def test_many_groups():
    e, T = 2047, 5000
    values = [0] + sorted(np.random.RandomState(1).randint(0, T + 1, e - 1).tolist()) + [T]
    x, w = operands("fwd", T, 16, 32, e)
    y, s = reference("fwd", x, w, groups(values, T))
    assert ((call("fwd", x, w, offsets(values)).double() - y).abs() <= bound(y, s, 32, b.OUT_BF16)).all()
    dy, x = operands("wgrad", T, 16, 32, e)
    y, s = reference("wgrad", dy, x, groups(values, T))
    assert ((call("wgrad", dy, x, offsets(values), dt=b.OUT_F32).double() - y).abs() <= bound(y, s, 32, b.OUT_F32)).all()


def test_offsets_beyond_32_bits_of_elements():
    # a token matrix of more than 2^31 elements; its last groups
    T, k, n = 270_000, 8192, 24
    x = torch.zeros(T, k, dtype=torch.bfloat16, device="cuda")
    x[-400:] = randn(1, 400, k)
    w = rows16(randn(2, 2 * n, k) * 0.05)
    values = [T - 400, T - 137, T]
    y, s = reference("fwd", x[-400:], w, [(0, 263), (263, 400)])
    got = call("fwd", x, w, offsets(values), dt=b.OUT_F32)
    assert ((got[-400:].double() - y).abs() <= bound(y, s, k, b.OUT_F32)).all() and not got[:-400].any()
    dy = torch.zeros(T, n, dtype=torch.bfloat16, device="cuda")
    dy[-400:] = randn(3, 400, n)
    y, s = reference("wgrad", dy[-400:], x[-400:], [(0, 263), (263, 400)])
    assert ((call("wgrad", dy, x, offsets(values), dt=b.OUT_F32).double() - y).abs() <= bound(y, s, 263, b.OUT_F32)).all()
    got = call("dgrad", dy, w, offsets(values))
    y, s = reference("dgrad", dy[-400:], w, [(0, 263), (263, 400)])
    assert ((got[-400:].double() - y).abs() <= bound(y, s, n, b.OUT_BF16)).all()


def test_captured_and_on_another_stream():
    T, n, k, values = 900, 304, 264, [0, 1, 400, 400, 900]
    x, w = operands("fwd", T, n, k, 4)
    dy, _ = operands("wgrad", T, n, k, 4, 5)
    offs, ws = offsets(values), b.alloc_workspace("cuda")

    def body():
        y = call("fwd", x, w, offs, ws=ws)
        return y, call("dgrad", y, w, offs, ws=ws), call("wgrad", dy, x, offs, dt=b.OUT_F32, ws=ws)

    eager = [t.clone() for t in body()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on_side = [call("fwd", x, w, offs, ws=ws, stream=side), call("wgrad", dy, x, offs, dt=b.OUT_F32, ws=ws, stream=side)]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(on_side[0], eager[0]) and torch.equal(on_side[1], eager[2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = body()
    kept, kept_offs = x.clone(), offs.clone()
    x.zero_()
    offs.copy_(offsets([0, 0, 0, 0, 0]))                    # boundaries are read when the graph runs
    graph.replay()
    torch.cuda.synchronize()
    assert not captured[0].any() and not captured[2].any()
    x.copy_(kept)
    offs.copy_(kept_offs)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(c, e) for c, e in zip(captured, eager)) and b.fp4q_workspace_status(ws) == 0


def test_captured_with_contractions_in_parts():
    T, n, k, values = 12000, 130, 72, [0, 11000, 11000, 12000]
    dy, x = operands("wgrad", T, n, k, 3)
    offs, ws, scratch = offsets(values), b.alloc_workspace("cuda"), b.alloc_ragged_wgrad_scratch(T, n, k, 3, "cuda")
    want = call("wgrad", dy, x, offs, dt=b.OUT_F32, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call("wgrad", dy, x, offs, dt=b.OUT_F32, ws=ws, scratch=scratch)
    for _ in range(3):
        got.zero_()
        scratch.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and b.fp4q_workspace_status(ws) == 0


def test_a_wait_that_runs_out_is_reported():
    for T, e in ((4000, 1), (100, 4)):                      # pairs and single CTAs, whose first one always has a tile
        values = [0] + [T * (i + 1) // e for i in range(e)]
        for op in ("fwd", "wgrad"):
            a, w = operands(op, T, 300, 520, e)
            ws = b.alloc_workspace("cuda")
            want = call(op, a, w, offsets(values), ws=ws)
            b.fp4q_workspace_set_wait_limit(ws, 2000)
            b.fp4q_debug_withhold_load(ws, 2 if op == "fwd" or T > 100 else 1)
            call(op, a, w, offsets(values), ws=ws)
            assert b.fp4q_workspace_status(ws) == 7
            b.fp4q_debug_withhold_load(ws, 0)
            b.fp4q_workspace_set_wait_limit(ws, 0)
            assert torch.equal(call(op, a, w, offsets(values), ws=ws), want) and b.fp4q_workspace_status(ws) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_layer_and_its_gradients(dtype):
    T, n, k, values = 300, 72, 100, [0, 50, 50, 180, 290]
    offs, spans = offsets(values), groups(values, T)
    x, w = randn(1, T, k).to(dtype).requires_grad_(), (randn(2, 4, n, k) * 0.1).to(dtype).requires_grad_()
    y = autograd.ragged_linear(x, w, offs)
    dy = randn(3, T, n).to(torch.bfloat16)
    y.backward(dy)
    xb, wb = x.detach().bfloat16().double(), w.detach().bfloat16().double()
    for g, (i, j) in enumerate(spans):
        want = [xb[i:j] @ wb[g].T, dy[i:j].double() @ wb[g], dy[i:j].double().T @ xb[i:j]]
        scale = [xb[i:j].abs() @ wb[g].abs().T, dy[i:j].double().abs() @ wb[g].abs(), dy[i:j].double().abs().T @ xb[i:j].abs()]
        for got, u, s in zip([y[i:j], x.grad[i:j], w.grad[g]], want, scale):
            assert ((got.double() - u).abs() <= u.abs() * 2 ** -8 + s * 20 * 2 ** -22).all()
    assert not y[290:].any() and not x.grad[290:].any() and x.grad.dtype == dtype and w.grad.dtype == dtype
    # against differences: y is linear in either, so a step of any size will do
    d = randn(4, T, k).to(torch.bfloat16)
    moved = autograd.ragged_linear(d.to(dtype), w.detach(), offs)
    lhs, rhs = (moved.double() * dy.double()).sum(), (x.grad.double() * d.double()).sum()
    assert abs(lhs - rhs) <= 2 ** -8 * ((moved.double() * dy.double()).abs().sum() + (x.grad.double() * d.double()).abs().sum())
