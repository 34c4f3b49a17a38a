"""Timed cases of the operators around an expert stack's training step that work on 16-bit and FP32 tensors: the BF16 products of
groups of any size (forward, input gradient, weight gradient) and the orthogonalised update of the weights they belong to.

`run` computes a pass in plain torch operations, in FP32, or, with `own`, through the calls of paper_2607_24953_b200.binding.

  ragged products   Y_t = W_g X_t,  dX_t = W_g^T dY_t,  dW_g = sum over t of dY_t X_t^T,  for the rows t of group g; groups start anywhere and
                    may be empty, rows behind the last group are nobody's and stay as they were
  newton_schulz     M <- beta M + G,  U = G + beta M (Nesterov) or M or, without a momentum, G;  X = U / (|U| + eps), then for every step
                    X <- a X + (b A + c A A) X with A = X X^T on the shorter side;  O = scale X in BF16; one matrix or a stack of them
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS, BETA, EPS = 5, 0.95, 1e-7


def listed():
    return [
        # The tiny linear layer's weight: five steps of products that take a microsecond or two each, so launches are all there is.
        _ns("update tiny", 1, 256, 256, "f32", True, True),
        # A down projection of the 1B-class model, wider than tall.
        _ns("update 1B", 1, 2048, 5632, "f32", True, True),
        # The largest matrix of the 7B-class model, taller than wide: the products are bound by the tensor cores.
        _ns("update 7B", 1, 11008, 4096, "f32", True, True),
        # The expert layer's stack of gradients as a BF16 weight gradient leaves it.
        _ns("update experts", 128, 768, 2048, "bf16", True, True),
        # A small stack of pruned, odd-sized matrices without a momentum of their own.
        _ns("update odd", 3, 1003, 777, "bf16", False, False),
        # Serving one token: eight rows for eight of 128 experts, bound by the weights that these experts have.
        _product("fwd token", "fwd", 8, 128, 768, 2048, "bf16", 0.0, 0),
        # A short prompt through odd-sized experts into an FP32 residual, in a buffer that is longer than the batch.
        _product("fwd odd", "fwd", 1999, 13, 1003, 2731, "f32", 0.8, 49),
        # The expert layer: 16384 tokens, eight experts each of 128, skewed loads.
        _product("fwd experts", "fwd", 131072, 128, 768, 2048, "bf16", 0.8, 0),
        # Its backward pass with respect to the tokens.
        _product("dgrad experts", "dgrad", 131072, 128, 768, 2048, "bf16", 0.8, 0),
        # A microbatch of a few hundred tokens through few experts.
        _product("dgrad odd", "dgrad", 1531, 8, 2731, 1003, "f32", 0.5, 7),
        # The stack's weight gradient in FP32, as a master weight's update wants it: groups of a few rows and of thousands.
        _product("wgrad experts", "wgrad", 131072, 128, 768, 2048, "f32", 0.8, 0),
        # A small batch: most of the experts got no or only a few tokens.
        _product("wgrad few", "wgrad", 300, 64, 1024, 512, "bf16", 1.2, 5),
    ]


def _ns(name, count, rows, cols, grad, momentum, nesterov):
    return {"name": name, "op": "ns", "count": count, "rows": rows, "cols": cols, "grad": grad, "momentum": momentum, "nesterov": nesterov}


def _product(name, op, rows, experts, n, k, out, skew, spare):
    """rows of token matrices for `experts` matrices of n x k; skew: of the loads (0 = even odds); spare: rows behind the last group."""
    return {"name": name, "op": op, "rows": rows, "experts": experts, "n": n, "k": k, "out": out, "skew": skew, "spare": spare, "load_seed": 7}


def _spread(rng, lo, hi):
    """A size between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most_ns, most_product = _ns_flops(1, 11008, 4096), 2.0 * 131072 * 768 * 2048
    while True:
        if rng.random() < 0.4:
            c = _ns("", _spread(rng, 1, 128), _spread(rng, 16, 11008), _spread(rng, 16, 11008), rng.choice(["f32", "bf16"]), rng.random() < 0.7, rng.random() < 0.7)
            if _ns_flops(c["count"], c["rows"], c["cols"]) > most_ns or c["count"] * c["rows"] * c["cols"] > 128 * 768 * 2048:
                continue
        else:
            op = rng.choice(["fwd", "dgrad", "wgrad"])
            c = _product("", op, _spread(rng, 1, 131072), _spread(rng, 1, 128), _spread(rng, 16, 11008), _spread(rng, 16, 11008), rng.choice(["bf16", "f32"]),
                         rng.choice([0.0, 0.5, 0.8, 1.2]), rng.choice([0, 0, 1, 33]))
            c["load_seed"] = rng.randrange(1 << 20)
            if 2.0 * c["rows"] * c["n"] * c["k"] > most_product or c["experts"] * c["n"] * c["k"] > 128 * 768 * 2048 or c["rows"] * max(c["n"], c["k"]) > 131072 * 2048:
                continue
        del c["name"]
        return c


def _ns_flops(count, rows, cols):
    """Multiplications and additions of all steps, those of symmetric products counted once for either half."""
    m, n = float(min(rows, cols)), float(max(rows, cols))
    return STEPS * count * (m * m * n + m * m * m + 2 * m * m * n)


def _loads(case):
    r = np.random.RandomState(case["load_seed"])
    p = r.permutation(np.arange(1, case["experts"] + 1, dtype=np.float64) ** -case["skew"])
    return r.multinomial(case["rows"], p / p.sum())


def work(case):
    if case["op"] == "ns":
        size = float(case["count"] * case["rows"] * case["cols"])
        return {"bytes": size * ((4 if case["grad"] == "f32" else 2) + (8 if case["momentum"] else 0) + 2), "flops": _ns_flops(case["count"], case["rows"], case["cols"])}
    t, n, k, e, wide = case["rows"], case["n"], case["k"], case["experts"], 4 if case["out"] == "f32" else 2
    used = int((_loads(case) > 0).sum())
    size = {"fwd": 2.0 * t * k + 2.0 * used * n * k + float(wide) * t * n,
            "dgrad": 2.0 * t * n + 2.0 * used * n * k + float(wide) * t * k,
            "wgrad": 2.0 * t * (n + k) + float(wide) * e * n * k}[case["op"]]
    return {"bytes": size + 8.0 * (e + 1), "flops": 2.0 * t * n * k}


def _gen(seed, j):
    return torch.Generator(DEVICE).manual_seed((seed * 16 + j) & 0x7FFFFFFFFFFF)


def _randn(seed, j, *shape):
    return torch.randn(*shape, generator=_gen(seed, j), device=DEVICE)


def _pitched(t):
    """A BF16 matrix in rows of whole 16 bytes."""
    buf = torch.zeros(t.shape[0], (t.shape[1] + 7) // 8 * 8, dtype=torch.bfloat16, device=DEVICE)
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


def _gradient(seed, j, case, scale):
    """Gradients of a weight matrix: half their rank in directions of falling strength, noise on top, some rows stronger than others."""
    e, m, n = case["count"], case["rows"], case["cols"]
    rank = max(1, min(m, n) // 2)
    strength = torch.arange(1, rank + 1, device=DEVICE, dtype=torch.float32) ** -0.5
    g = torch.matmul(_randn(seed, j, e, m, rank) * strength, _randn(seed, j + 1, e, rank, n))
    g += 0.5 * _randn(seed, j + 2, e, m, n)
    g *= torch.exp(0.5 * _randn(seed, j + 3, e, m, 1)) * scale
    return g


def prepare(case, seed):
    s = {"case": case}
    if case["op"] == "ns":
        g = _gradient(seed, 0, case, 1e-3).to(torch.float32 if case["grad"] == "f32" else torch.bfloat16)
        s["g"] = g[0] if case["count"] == 1 else g
        s["m"] = None
        if case["momentum"]:
            m = _gradient(seed, 4, case, 5e-3)
            s["m"] = m[0] if case["count"] == 1 else m
        s["scale"] = 0.2 * math.sqrt(max(case["rows"], case["cols"]))
        s["o"] = torch.zeros(s["g"].shape, dtype=torch.bfloat16, device=DEVICE)
        if own:
            from paper_2607_24953_b200 import binding
            s["scratch"] = binding.alloc_newton_schulz_scratch(case["count"], case["rows"], case["cols"], DEVICE)
            s["ws"] = binding.alloc_workspace(DEVICE)
        return s
    counts = _loads(case)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    t, n, k, e = case["rows"] + case["spare"], case["n"], case["k"], case["experts"]
    s["offsets"] = torch.from_numpy(offsets.astype(np.int64)).to(DEVICE)
    s["groups"] = [(g, int(offsets[g]), int(offsets[g + 1])) for g in range(e)]     # as the routing step that made the permutation knows them
    if case["op"] != "dgrad":
        s["x"] = _pitched(_randn(seed, 0, t, k) * torch.exp(0.5 * _randn(seed, 1, 1, k)))
    if case["op"] != "fwd":
        s["dy"] = _pitched(_randn(seed, 2, t, n) * torch.exp(_randn(seed, 3, t, 1)) * 1e-3)
    if case["op"] != "wgrad":
        s["w"] = _pitched(_randn(seed, 4, e * n, k) * 0.02)
    dtype = torch.float32 if case["out"] == "f32" else torch.bfloat16
    rows, cols = {"fwd": (t, n), "dgrad": (t, k), "wgrad": (e * n, k)}[case["op"]]
    s["out"] = torch.zeros(rows, (cols + 7) // 8 * 8, dtype=dtype, device=DEVICE)[:, :cols]
    if own:
        from paper_2607_24953_b200 import binding
        s["ws"] = binding.alloc_workspace(DEVICE)
    return s


def run(s):
    case = s["case"]
    if own:
        from paper_2607_24953_b200 import binding as b
        if case["op"] == "ns":
            o = b.fp4q_newton_schulz(s["g"], momentum=s["m"], beta=BETA, nesterov=case["nesterov"], coefficients=(COEFFICIENTS,) * STEPS, eps=EPS,
                                     scale=s["scale"], out=s["o"], scratch=s["scratch"], ws=s["ws"])
            return {"o": o, "m": s["m"]}
        dt = b.OUT_F32 if case["out"] == "f32" else b.OUT_BF16
        if case["op"] == "fwd":
            return b.fp4q_ragged_gemm_fwd(s["x"], s["w"], s["offsets"], out=s["out"], dt=dt, ws=s["ws"])
        if case["op"] == "dgrad":
            return b.fp4q_ragged_gemm_dgrad(s["dy"], s["w"], s["offsets"], out=s["out"], dt=dt, ws=s["ws"])
        return b.fp4q_ragged_gemm_wgrad(s["dy"], s["x"], s["offsets"], out=s["out"], dt=dt, ws=s["ws"])
    return _plain_ns(s, case) if case["op"] == "ns" else _plain_product(s, case)


def _plain_ns(s, case):
    g, m = s["g"].float(), s["m"]
    if m is not None:
        m.mul_(BETA).add_(g)
        u = g + BETA * m if case["nesterov"] else m
    else:
        u = g
    norm = torch.sqrt((u.double() * u.double()).sum(dim=(-2, -1), keepdim=True))
    x = u * (1.0 / (norm + EPS)).float()
    tall = case["rows"] > case["cols"]
    if tall:
        x = x.mT
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    o = (s["scale"] * (x.mT if tall else x)).to(torch.bfloat16)
    return {"o": o, "m": m}


def _plain_product(s, case):
    n, op = case["n"], case["op"]
    if op == "wgrad":
        return torch.cat([s["dy"][a:b].float().T @ s["x"][a:b].float() for _, a, b in s["groups"]]).to(s["out"].dtype)
    w = s["w"]
    if op == "fwd":
        rows = [s["x"][a:b].float() @ w[g * n:(g + 1) * n].float().T for g, a, b in s["groups"] if b > a]
    else:
        rows = [s["dy"][a:b].float() @ w[g * n:(g + 1) * n].float() for g, a, b in s["groups"] if b > a]
    return torch.cat(rows + [s["out"][case["rows"]:].float()]).to(s["out"].dtype)


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    if case["op"] == "ns":
        u, m = s["g"].double(), None
        if s["m"] is not None:
            m = s["g"].double() + BETA * s["m"].double()
            u = s["g"].double() + BETA * m if case["nesterov"] else m
        x = u / (torch.linalg.vector_norm(u, dim=(-2, -1), keepdim=True) + EPS)
        del u
        a, b, c = COEFFICIENTS
        wide = case["cols"] >= case["rows"]
        for _ in range(STEPS):
            q = torch.matmul(x, x.transpose(-1, -2)) if wide else torch.matmul(x.transpose(-1, -2), x)
            p = torch.matmul(q, c * q)
            p += b * q
            p.diagonal(dim1=-2, dim2=-1).add_(a)
            x = torch.matmul(p, x) if wide else torch.matmul(x, p)
        return {"o": x * s["scale"], "m": m}
    n, k, op = case["n"], case["k"], case["op"]
    if op == "wgrad":
        out = torch.zeros(case["experts"], n, k, dtype=torch.float64, device=DEVICE)
        for g, a, b in s["groups"]:
            torch.matmul(s["dy"][a:b].double().T, s["x"][a:b].double(), out=out[g])
        return out.view(-1, k)
    out = torch.zeros(case["rows"] + case["spare"], n if op == "fwd" else k, dtype=torch.float64, device=DEVICE)
    for g, a, b in s["groups"]:
        if b > a:
            w = s["w"][g * n:(g + 1) * n].double()
            out[a:b] = s["x"][a:b].double() @ w.T if op == "fwd" else s["dy"][a:b].double() @ w
    return out
