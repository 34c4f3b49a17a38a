"""Timed cases of the operators around a linear layer in 8 bits with a scale for every block of 128: the norm that feeds it, the quantizers, the three
products, and the clipping of the gradients that a step leaves.

`run` computes a pass in plain torch operations, in FP32, or, with `own`, through the calls of paper_2607_24953_b200.binding.

  rms_norm      h = x + residual, rounded to the residual's type;  r = 1 / sqrt(mean(h^2) + eps);  y = h r weight, in BF16 and/or 8 bits
  rms_norm_bwd  g = dy weight;  dx = r (g - h r mean(g h r)) + dh;  dweight = sum over rows of dy h r
  fp8_quantize  S = max(M, 2^-100) / 448 for the largest magnitude M of 128 elements of a row (1D blocks; the transpose in blocks of its own) or of
                128 x 128 (square ones, the transpose shares them);  q = x / S in E4M3
  fp8 products  Y = X^ W^^T,  dX = dY^ W^,  dW = dY^^T X^:  X and dY in 1D blocks along the contraction, W in square ones
  clip          norm = sqrt(sum of squares over all tensors);  out = g min(1, max_norm / (norm + 1e-6))
"""
import math

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-6
BLOCK, MX, TOP = 128, 32, 448.0
LEAST = 2.0 ** -100


def listed():
    return [
        # Serving one token: the norm before the query and key projections, written as their MXFP8 operand.  Launches and latency are all there is.
        _norm("norm token", "fwd", 1, 4096, "bf16", "mxfp8", True),
        # Training the 7B-class model: residual stream in BF16, output in 8 bits for the product and in BF16 for the weight gradient.
        _norm("norm 7B", "fwd", 16384, 4096, "bf16", "fp8", True),
        # Its backward pass, with the gradient that comes along the residual stream.
        _norm("norm bwd 7B", "bwd", 16384, 4096, "bf16", "", True),
        # An odd width on an FP32 residual stream, a packed batch of odd length.
        _norm("norm bwd odd", "bwd", 1999, 2731, "f32", "", True),
        # An output gradient of the 7B-class model: one reading gives the operands of both backward products.
        _quantize("quantize gradient", 16384, 4096, "bf16", False),
        # An FP32 master weight of odd size, both orientations under one set of scales.
        _quantize("quantize weight odd", 1003, 2731, "f32", True),
        # Serving one token through the 7B-class down projection: bound by the weight's bytes.
        _product("fp8 token", "fwd", 1, 4096, 11008, "bf16"),
        # The gate projection of the 7B-class model, forward: bound by the tensor cores.
        _product("fp8 fwd 7B", "fwd", 16384, 11008, 4096, "bf16"),
        # A microbatch of odd length through an odd-sized layer, backward into an FP32 stream.
        _product("fp8 dgrad odd", "dgrad", 1999, 1003, 2731, "f32"),
        # A weight gradient in FP32: the contraction runs over all tokens, both operands in 1D blocks.
        _product("fp8 wgrad 7B", "wgrad", 16384, 4096, 4096, "f32"),
        # The gradients of two tiny layers and their norms: a few small tensors, so launches are all there is.
        _clip("clip tiny", 2, 256, 256, "bf16", "bf16"),
        # The FP32 gradients of a block of the 7B-class model, clipped into the BF16 tensors that the orthogonalised update reads.
        _clip("clip 7B", 1, 4096, 11008, "f32", "bf16"),
    ]


def _norm(name, op, rows, cols, stream, q, residual):
    """stream: the type of the residual stream; q: the 8-bit output's format; residual: whether there is one (backward: a gradient along it)."""
    return {"name": name, "op": "norm_" + op, "rows": rows, "cols": cols, "stream": stream, "q": q, "residual": residual}


def _quantize(name, rows, cols, dtype, square):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "square": square}


def _product(name, op, t, n, k, out):
    return {"name": name, "op": op, "t": t, "n": n, "k": k, "out": out}


def _clip(name, blocks, hidden, ffn, dtype, out):
    """blocks of four hidden x hidden matrices, three of hidden x ffn and two vectors."""
    return {"name": name, "op": "clip", "blocks": blocks, "hidden": hidden, "ffn": ffn, "dtype": dtype, "out": out}


def _spread(rng, lo, hi):
    """A size between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["norm_fwd", "norm_fwd", "norm_bwd", "quantize", "quantize", "fwd", "fwd", "dgrad", "wgrad", "clip"])
        if op.startswith("norm"):
            c = _norm("", op[5:], _spread(rng, 1, 16384), _spread(rng, 16, 16384), rng.choice(["bf16", "f32"]), rng.choice(["", "mxfp8", "fp8"]), rng.random() < 0.7)
            if op == "norm_bwd":
                c["q"] = ""
            if c["rows"] * c["cols"] > 16384 * 4096:
                continue
        elif op == "quantize":
            c = _quantize("", _spread(rng, 1, 16384), _spread(rng, 1, 11008), rng.choice(["bf16", "f32"]), rng.random() < 0.5)
            if c["rows"] * c["cols"] > 16384 * 4096:
                continue
        elif op == "clip":
            c = _clip("", _spread(rng, 1, 6), _spread(rng, 16, 4096), _spread(rng, 16, 11008), rng.choice(["bf16", "f32"]), rng.choice(["bf16", "f32"]))
            if sum(a * b for a, b in _shapes(c)) > 4 * 4096 * 4096 + 3 * 4096 * 11008:
                continue
        else:
            c = _product("", op, _spread(rng, 1, 16384), _spread(rng, 16, 11008), _spread(rng, 16, 11008), rng.choice(["bf16", "f32"]))
            if c["t"] * c["n"] * c["k"] > 16384 * 11008 * 4096:
                continue
        del c["name"]
        return c


def _shapes(case):
    h, f = case["hidden"], case["ffn"]
    return ([(h, h)] * 4 + [(f, h)] * 2 + [(h, f)] + [(1, h)] * 2) * case["blocks"]


def _bytes(dtype):
    return 4 if dtype == "f32" else 2


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def work(case):
    op = case["op"]
    if op.startswith("norm"):
        r, c, wide = float(case["rows"]), float(case["cols"]), _bytes(case["stream"])
        if op == "norm_bwd":
            return {"bytes": r * c * (2 + 2 * wide + (wide if case["residual"] else 0)) + 4 * r + 8 * c, "flops": 8 * r * c}
        read = 2 + 2 * wide if case["residual"] else wide      # a residual's sum is written as well
        q = {"": 2.0, "mxfp8": 1 + 1 / 32, "fp8": 3 + 4 / 128}[case["q"]]
        return {"bytes": r * c * (read + q) + 4 * r + 4 * c, "flops": 6 * r * c}
    if op == "quantize":
        r, c = case["rows"], case["cols"]
        scales = _blocks(r) * _blocks(c) if case["square"] else r * _blocks(c) + c * _blocks(r)
        return {"bytes": float(r * c * (_bytes(case["dtype"]) + 2) + 4 * scales), "flops": 4.0 * r * c}
    if op == "clip":
        n = float(sum(a * b for a, b in _shapes(case)))
        return {"bytes": n * (_bytes(case["dtype"]) + _bytes(case["out"])), "flops": 3 * n}
    t, n, k, wide = float(case["t"]), float(case["n"]), float(case["k"]), _bytes(case["out"])
    size = {"fwd": t * k + n * k + wide * t * n, "dgrad": t * n + n * k + wide * t * k, "wgrad": t * (n + k) + wide * n * k}[op]
    return {"bytes": size, "flops": 2 * t * n * k}


def _gen(seed, j):
    return torch.Generator(DEVICE).manual_seed((seed * 64 + j) & 0x7FFFFFFFFFFF)


def _randn(seed, j, *shape):
    return torch.randn(*shape, generator=_gen(seed, j), device=DEVICE)


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _pitched(t):
    """t in rows of whole 16 bytes."""
    per = 16 // t.element_size()
    buf = torch.zeros(t.shape[0], (t.shape[1] + per - 1) // per * per, dtype=t.dtype, device=DEVICE)
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


def _activations(seed, j, rows, cols):
    """Heavy-tailed rows, and every two hundredth channel much larger than the others."""
    x = _randn(seed, j, rows, cols) * torch.exp(0.5 * _randn(seed, j + 1, rows, cols))
    return x * torch.where(torch.rand(1, cols, generator=_gen(seed, j + 2), device=DEVICE) < 0.005, 30.0, 1.0)


def _gradients(seed, j, rows, cols):
    """Rows of very different size, as tokens' gradients are."""
    return _randn(seed, j, rows, cols) * torch.exp(1.5 * _randn(seed, j + 1, rows, 1)) * 1e-3


def _in_blocks(x, down, along):
    """x padded with zeros and cut: [row blocks, down, column blocks, along]."""
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, -c % along, 0, -r % down))
    return x.reshape((r + down - 1) // down, down, (c + along - 1) // along, along)


def _codes(x, down):
    """(E4M3 codes, FP32 scales of blocks of down x 128) of x in FP32."""
    b = _in_blocks(x, down, BLOCK)
    scale = b.abs().amax(dim=(1, 3), keepdim=True).clamp_min(LEAST) / TOP
    q = (b / scale).clamp(-TOP, TOP).to(torch.float8_e4m3fn)
    return q.reshape(q.shape[0] * down, -1)[:x.shape[0], :x.shape[1]], scale[:, 0, :, 0]


def _values(q, scale, down):
    """What codes and scales stand for, in the scales' type."""
    r, c = q.shape
    return q.to(scale.dtype) * scale.repeat_interleave(down, 0)[:r].repeat_interleave(BLOCK, 1)[:, :c]


def _mx_codes(x):
    """(E4M3 codes, UE8M0 scales of 32 elements of a row) of x in FP32: the smallest power of two S with 448 S >= M, not below 2^-127."""
    b = _in_blocks(x, 1, MX)
    top = b.abs().amax(dim=3, keepdim=True).double()
    m, e = torch.frexp(top / TOP)                       # M / 448 = m 2^e, m in [1/2, 1)
    e = torch.where(top > 0, torch.where(m == 0.5, e - 1, e), -127).clamp(-127, 127)
    q = (b.double() * torch.exp2(-e.double())).float().clamp(-TOP, TOP).to(torch.float8_e4m3fn)
    return q.reshape(x.shape[0], -1)[:, :x.shape[1]], (e + 127)[:, 0, :, 0].to(torch.uint8)


def prepare(case, seed):
    s, op = {"case": case}, case["op"]
    if own:
        from paper_2607_24953_b200 import binding as b
        s["ws"] = b.alloc_workspace(DEVICE)
    if op.startswith("norm"):
        rows, cols, stream = case["rows"], case["cols"], _type(case["stream"])
        s["weight"] = 1 + 0.2 * _randn(seed, 0, cols)
        if op == "norm_fwd":
            if case["residual"]:
                s["x"] = _randn(seed, 1, rows, cols).to(torch.bfloat16)
                s["residual"] = _pitched(_activations(seed, 2, rows, cols).to(stream))
            else:
                s["x"], s["residual"] = _activations(seed, 2, rows, cols).to(stream), None
            if own:
                fmt = {"": b.Q_NONE, "mxfp8": b.Q_MXFP8, "fp8": b.Q_FP8}[case["q"]]
                s["out"] = b.alloc_norm(s["x"], s["residual"], y=case["q"] != "mxfp8", q=fmt, rstd=True)
        else:
            s["h"] = _pitched(_activations(seed, 2, rows, cols).to(stream))
            s["rstd"] = torch.rsqrt(s["h"].float().square().mean(1) + EPS)
            s["dy"] = _pitched(_gradients(seed, 5, rows, cols).to(torch.bfloat16))
            s["dh"] = _pitched(_gradients(seed, 7, rows, cols).to(stream)) if case["residual"] else None
            if own:
                s["dx"] = torch.empty_like(s["h"])
                s["dweight"] = torch.empty(cols, device=DEVICE)
                s["scratch"] = b.alloc_rms_norm_scratch(rows, cols, DEVICE)
        return s
    if op == "quantize":
        x = (_randn(seed, 0, case["rows"], case["cols"]) * 0.02) if case["square"] else _gradients(seed, 0, case["rows"], case["cols"])
        s["x"] = _pitched(x.to(_type(case["dtype"])))
        if own:
            s["out"] = b.alloc_fp8tensor(case["rows"], case["cols"], DEVICE, square=case["square"])
        return s
    if op == "clip":
        s["g"] = [(_randn(seed, j, *shape) * 1e-3 * (1 + j % 3)).to(_type(case["dtype"])) for j, shape in enumerate(_shapes(case))]
        n = sum(g.numel() for g in s["g"])
        s["max_norm"] = 1e-3 * math.sqrt(n)                # about half of the norm: it has to be clipped
        s["out"] = [torch.empty(g.shape, dtype=_type(case["out"]), device=DEVICE) for g in s["g"]]
        if own:
            s["scratch"] = b.alloc_global_norm_scratch(s["g"])
        return s
    t, n, k = case["t"], case["n"], case["k"]
    # The operands' codes as the contraction runs: [rows, contraction] each, as the quantizers leave them.
    a = {"fwd": lambda: _activations(seed, 0, t, k), "dgrad": lambda: _gradients(seed, 0, t, n), "wgrad": lambda: _gradients(seed, 0, t, n).T}[op]().to(torch.bfloat16).float()
    w = {"fwd": lambda: _randn(seed, 4, n, k) * 0.02, "dgrad": lambda: (_randn(seed, 4, n, k) * 0.02).T, "wgrad": lambda: _activations(seed, 4, t, k).T}[op]().float()
    for name, m, down in (("a", a, 1), ("b", w, 1 if op == "wgrad" else BLOCK)):
        q, scale = _codes(m, down)
        s[name], s[name + "_scale"] = _pitched(q.contiguous().view(torch.uint8)), scale.contiguous()
    s["out"] = _pitched(torch.zeros(a.shape[0], w.shape[0], dtype=_type(case["out"]), device=DEVICE))
    if own:
        x, y, sx, sy = s["a"], s["b"], s["a_scale"], s["b_scale"]
        if op == "fwd":
            s["A"], s["B"] = b.Fp8Tensor(t, k, x, sx), b.Fp8Tensor(n, k, y, sy, square=True)
        elif op == "dgrad":
            s["A"], s["B"] = b.Fp8Tensor(t, n, x, sx), b.Fp8Tensor(n, k, None, sy.T.contiguous(), y, square=True)
        else:
            s["A"], s["B"] = b.Fp8Tensor(t, n, None, None, x, sx), b.Fp8Tensor(t, k, None, None, y, sy)
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2607_24953_b200 import binding as b
        if op == "norm_fwd":
            return _norm_outputs(s["case"], b.fp4q_rms_norm(s["x"], s["weight"], s["residual"], eps=EPS, out=s["out"]))
        if op == "norm_bwd":
            dx, dw = b.fp4q_rms_norm_bwd(s["dy"], s["h"], s["rstd"], s["weight"], dh=s["dh"], out=s["dx"], dweight=s["dweight"], scratch=s["scratch"])
            return {"dx": dx, "dweight": dw}
        if op == "quantize":
            q = b.fp4q_fp8_quantize(s["x"], out=s["out"], square=s["case"]["square"])
            r, c = s["case"]["rows"], s["case"]["cols"]
            return {"q": q.q[:, :c].view(torch.float8_e4m3fn), "scale": q.scale, "q_t": q.q_t[:, :r].view(torch.float8_e4m3fn), "scale_t": q.scale_t}
        if op == "clip":
            norm = b.fp4q_clip_grad_norm(s["g"], s["max_norm"], outs=s["out"], scratch=s["scratch"])
            return {"norm": norm, "g": s["out"]}
        dt = b.OUT_F32 if s["case"]["out"] == "f32" else b.OUT_BF16
        call = {"fwd": b.fp4q_fp8_gemm_fwd, "dgrad": b.fp4q_fp8_gemm_dgrad, "wgrad": b.fp4q_fp8_gemm_wgrad}[op]
        return call(s["A"], s["B"], out=s["out"], dt=dt, ws=s["ws"])
    return {"norm_fwd": _plain_norm, "norm_bwd": _plain_norm_bwd, "quantize": _plain_quantize, "clip": _plain_clip}.get(op, _plain_product)(s)


def _norm_outputs(case, o):
    """The 8-bit output as what its bytes are."""
    d = {"h": o.h, "y": o.y, "rstd": o.rstd, "q": None, "scale": None}
    if case["q"]:
        d["q"] = o.q[:, :case["cols"]].view(torch.float8_e4m3fn)
        d["scale"] = o.scale.view(torch.float8_e8m0fnu) if case["q"] == "mxfp8" else o.scale
    return d


def _plain_norm(s):
    case = s["case"]
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["residual"].dtype)
    f = h.float()
    rstd = torch.rsqrt(f.square().mean(1) + EPS)
    y = f * rstd[:, None] * s["weight"]
    q, scale = {"": lambda _: (None, None), "mxfp8": _mx_codes, "fp8": lambda v: _codes(v, 1)}[case["q"]](y)
    return {"h": h if s["residual"] is not None else None, "y": y.to(torch.bfloat16) if case["q"] != "mxfp8" else None, "rstd": rstd, "q": q,
            "scale": scale.view(torch.float8_e8m0fnu) if case["q"] == "mxfp8" else scale}


def _plain_norm_bwd(s):
    x = s["h"].float() * s["rstd"][:, None]
    dy = s["dy"].float()
    g = dy * s["weight"]
    dx = s["rstd"][:, None] * (g - x * (g * x).mean(1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(s["h"].dtype), "dweight": (dy * x).sum(0)}


def _plain_quantize(s):
    x, square = s["x"].float(), s["case"]["square"]
    q, scale = _codes(x, BLOCK if square else 1)
    q_t, scale_t = (q.T.contiguous(), None) if square else _codes(x.T, 1)
    return {"q": q, "scale": scale, "q_t": q_t, "scale_t": scale_t}


def _plain_clip(s):
    norm = torch.sqrt(torch.stack([g.double().square().sum() for g in s["g"]]).sum()).float()
    c = torch.clamp(s["max_norm"] / (norm + EPS), max=1.0)
    return {"norm": norm, "g": [(g.float() * c).to(o.dtype) for g, o in zip(s["g"], s["out"])]}


def _plain_product(s):
    down = 1 if s["case"]["op"] == "wgrad" else BLOCK
    a = _values(s["a"].view(torch.float8_e4m3fn), s["a_scale"], 1)
    b = _values(s["b"].view(torch.float8_e4m3fn), s["b_scale"], down)
    return (a @ b.T).to(s["out"].dtype)


def exact(case, seed):
    """The definitions in 64 bits; 8-bit codes as the quotients that they are rounded from."""
    s, op = prepare(case, seed), case["op"]
    if op == "norm_fwd":
        h = s["x"].double()
        if s["residual"] is not None:
            h = h + s["residual"].double()
        f = h if s["residual"] is None else h.to(s["residual"].dtype).double()
        rstd = 1 / torch.sqrt((f * f).sum(1) / case["cols"] + EPS)
        y = f * s["weight"].double() * rstd[:, None]
        q = scale = None
        if case["q"]:
            n = BLOCK if case["q"] == "fp8" else MX
            top = torch.nn.functional.pad(y, (0, -case["cols"] % n)).abs().unflatten(1, (-1, n)).amax(2)
            scale = top.clamp_min(LEAST) / TOP if case["q"] == "fp8" else torch.exp2(torch.ceil(torch.log2(top / TOP)).clamp_min(-127))
            q = y / scale.repeat_interleave(n, 1)[:, :case["cols"]]
        return {"h": h if s["residual"] is not None else None, "y": y if case["q"] != "mxfp8" else None, "rstd": rstd, "q": q, "scale": scale}
    if op == "norm_bwd":
        h, dy, w = s["h"].double(), s["dy"].double(), s["weight"].double()
        r = s["rstd"].double()[:, None]
        dot = (dy * w * h).sum(1, keepdim=True) / case["cols"]
        dx = r * dy * w - r * r * r * dot * h
        if s["dh"] is not None:
            dx += s["dh"].double()
        return {"dx": dx, "dweight": torch.einsum("tc,tc->c", dy * r, h)}
    if op == "quantize":
        x = s["x"].double()
        if case["square"]:
            p = torch.nn.functional.pad(x.abs(), (0, -case["cols"] % BLOCK, 0, -case["rows"] % BLOCK))
            scale = p.unflatten(0, (-1, BLOCK)).unflatten(2, (-1, BLOCK)).amax((1, 3)).clamp_min(LEAST) / TOP
            q = x / scale.repeat_interleave(BLOCK, 0)[:case["rows"]].repeat_interleave(BLOCK, 1)[:, :case["cols"]]
            return {"q": q, "scale": scale, "q_t": q.T.contiguous(), "scale_t": None}
        d = {}
        for name, m in (("", x), ("_t", x.T)):
            scale = torch.nn.functional.pad(m.abs(), (0, -m.shape[1] % BLOCK)).unflatten(1, (-1, BLOCK)).amax(2).clamp_min(LEAST) / TOP
            d["q" + name], d["scale" + name] = m / scale.repeat_interleave(BLOCK, 1)[:, :m.shape[1]], scale
        return d
    if op == "clip":
        g = [t.double() for t in s["g"]]
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(t) for t in g]))
        c = min(1.0, s["max_norm"] / (float(norm) + EPS))
        return {"norm": norm, "g": [t * c for t in g]}
    a = s["a"].view(torch.float8_e4m3fn).double() * s["a_scale"].double().repeat_interleave(BLOCK, 1)[:, :s["a"].shape[1]]
    b = s["b"].view(torch.float8_e4m3fn).double() * s["b_scale"].double().repeat_interleave(BLOCK, 1)[:, :s["b"].shape[1]] if op == "wgrad" else (
        s["b"].view(torch.float8_e4m3fn).double() * torch.kron(s["b_scale"].double(), torch.ones(BLOCK, BLOCK, dtype=torch.float64, device=DEVICE))[:s["b"].shape[0], :s["b"].shape[1]])
    return a @ b.T
