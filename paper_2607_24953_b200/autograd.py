"""Straight-through FP4 linear layer on top of the C-ABI calls (glue only; every step runs in the library's kernels).

Section 3.1 of the paper: the forward product uses 2D-block-quantized weights and activations (round to nearest),
the backward pass quantizes the incoming gradient once (stochastic rounding) and uses it, with the quantized
operands saved by the forward pass, in both backward products; the quantizers are treated as identity when
differentiating (straight-through estimator).  Because the blocks are 32x32, the transposed payloads the backward
products need are written by the same quantization call: nothing is re-quantized between forward and backward.
"""
from __future__ import annotations

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import binding


class _FP4LinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, seed, tensor_id, ws):
        # x [T, K], weight [N, K]; both are quantized once, with both payload layouts
        qx = binding.fp4q_quantize2d(x.to(torch.bfloat16).contiguous(), mode=binding.ROUND_NEAREST)
        qw = binding.fp4q_quantize2d(weight.to(torch.bfloat16).contiguous(), mode=binding.ROUND_NEAREST)
        y = binding.fp4q_gemm_fwd(qx, qw, dt=binding.OUT_BF16, ws=ws)
        ctx.qx, ctx.qw, ctx.ws = qx, qw, ws
        ctx.seed, ctx.tensor_id = int(seed), int(tensor_id)
        ctx.x_dtype, ctx.w_dtype = x.dtype, weight.dtype
        return y if y.is_contiguous() else y.contiguous()

    @staticmethod
    def backward(ctx, dy):
        qdy = binding.fp4q_quantize2d(dy.to(torch.bfloat16).contiguous(), mode=binding.ROUND_STOCHASTIC,
                                      seed=ctx.seed, tensor_id=ctx.tensor_id)
        dx = dw = None
        if ctx.needs_input_grad[0]:
            dx = binding.fp4q_gemm_dgrad(qdy, ctx.qw, dt=binding.OUT_BF16, ws=ctx.ws).to(ctx.x_dtype)
        if ctx.needs_input_grad[1]:
            dw = binding.fp4q_gemm_wgrad(qdy, ctx.qx, dt=binding.OUT_F32, ws=ctx.ws).to(ctx.w_dtype)
        ctx.qx = ctx.qw = None
        return dx, dw, None, None, None


_TENSORS = (torch.Tensor, torch.nn.Parameter)


def _find_observers():
    """A function that says whether anything looks into Python autograd functions just now: tracers, transforms, modes, forward-mode
    levels.  None where this torch lacks one of the names, which are not public."""
    try:
        compiling, tracing = torch.compiler.is_compiling, torch._C._get_tracing_state
        transforms, dispatch, function = torch._C._functorch.peek_interpreter_stack, torch._C._len_torch_dispatch_stack, torch._C._len_torch_function_stack
        forward_ad._current_level   # a variable: read at every call
    except AttributeError:
        return None

    def observed() -> bool:
        return (compiling() or transforms() is not None or dispatch() != 0 or function() != 0 or tracing() is not None
                or forward_ad._current_level >= 0)
    return observed


_observed = _find_observers()


def _plain(x, weight) -> bool:
    """Ordinary tensors on one GPU and nothing that looks into a Python autograd function: the native node does the same in half
    the host's time.  Everything else, what is refused included, goes through _FP4LinearFn."""
    return (_observed is not None and type(x) in _TENSORS and type(weight) in _TENSORS and x.is_cuda and weight.dim() == 2
            and x.device == weight.device and not _observed())


def _linear(x, weight, seed, tensor_id, ws):
    if _plain(x, weight):
        return binding._host().linear(x, weight, int(seed), int(tensor_id), ws)
    return _FP4LinearFn.apply(x, weight, seed, tensor_id, ws)


def fp4_linear(x: torch.Tensor, weight: torch.Tensor, seed: int = 0, tensor_id: int = 0, ws=None) -> torch.Tensor:
    """y = x^ weight^^T with FP4 forward and backward products.  x [..., K] and weight [N, K] live on the GPU;
    `seed` / `tensor_id` key the stochastic rounding of the incoming gradient (change one of them every step)."""
    if ws is None:
        ws = binding.alloc_workspace(x.device)
    if x.dim() == 2 and x.shape[1] != 0:   # nothing to fold: two autograd nodes less (reshape refuses rows of nothing)
        return _linear(x, weight, seed, tensor_id, ws)
    lead = x.shape[:-1]
    y = _linear(x.reshape(-1, x.shape[-1]), weight, seed, tensor_id, ws)
    return y.reshape(*lead, weight.shape[0])


class _RaggedLinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, row_offsets, ws):
        e, n, k = weight.shape
        xb, wb = _rows16(x), _rows16(weight.reshape(e * n, k))
        ctx.save_for_backward(xb, wb, row_offsets)
        ctx.ws, ctx.shape, ctx.x_dtype, ctx.w_dtype = ws, (e, n, k), x.dtype, weight.dtype
        return binding.fp4q_ragged_gemm_fwd(xb, wb, row_offsets, ws=ws).contiguous()

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        xb, wb, row_offsets = ctx.saved_tensors
        dyb, dx, dw = _rows16(dy), None, None
        if ctx.needs_input_grad[0]:
            dx = binding.fp4q_ragged_gemm_dgrad(dyb, wb, row_offsets, dt=_out16(ctx.x_dtype), ws=ctx.ws).to(ctx.x_dtype)
        if ctx.needs_input_grad[1]:
            dw = binding.fp4q_ragged_gemm_wgrad(dyb, xb, row_offsets, dt=_out16(ctx.w_dtype), ws=ctx.ws).to(ctx.w_dtype).reshape(ctx.shape)
        return dx, dw, None, None


def _out16(dtype: torch.dtype) -> int:
    """The type a gradient is computed in: not less than what it belongs to holds."""
    return binding.OUT_BF16 if dtype == torch.bfloat16 else binding.OUT_F32


def _rows16(t: torch.Tensor) -> torch.Tensor:
    """t in BF16 and in rows that start on 16 bytes, as the products read them; t itself where it is so."""
    t = t.to(torch.bfloat16)
    rows, cols = t.shape
    if t.stride(1) == 1 and t.stride(0) % 8 == 0 and t.stride(0) >= cols and t.data_ptr() % 16 == 0:
        return t
    out = torch.empty((rows, (cols + 7) // 8 * 8), dtype=torch.bfloat16, device=t.device)[:, :cols]
    return out.copy_(t)


def ragged_linear(x: torch.Tensor, weight: torch.Tensor, row_offsets: torch.Tensor, ws=None) -> torch.Tensor:
    """y_t = weight[g] x_t for the rows t of group g, in BF16: the expert layer as it is without FP4, on groups of any size.  x [T, K], weight
    [E, N, K], row_offsets int64 [E+1], non-decreasing, all on one GPU; rows that no group owns give zeros and get no gradient.  Gradients are
    computed in BF16 for BF16 tensors and in FP32 for others.  Differentiable once.  A backward pass that is captured into a CUDA graph needs, as with torch's own layers, leaves that no living eager graph holds."""
    if x.dim() != 2 or weight.dim() != 3 or x.shape[1] != weight.shape[2]:
        raise ValueError(f"x must be [T, K] and weight [E, N, K], not {list(x.shape)} and {list(weight.shape)}")
    if row_offsets.dim() != 1 or row_offsets.shape[0] != weight.shape[0] + 1:
        raise ValueError(f"row_offsets must hold one offset more than weight has groups, {weight.shape[0] + 1}, not {list(row_offsets.shape)}")
    if ws is None:
        ws = binding.alloc_workspace(x.device)
    return _RaggedLinearFn.apply(x, weight, row_offsets, ws)


class FP4Linear(torch.nn.Module):
    """Bias-free linear layer with an FP32 master weight and FP4 products.  Each backward pass draws fresh
    stochastic-rounding bits: the module counts its forward calls and uses the count as the Philox tensor id's
    high part, `layer_id` as the low 8 bits."""

    def __init__(self, in_features: int, out_features: int, layer_id: int = 0, seed: int = 0, device="cuda"):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, device=device, dtype=torch.float32))
        torch.nn.init.normal_(self.weight, std=0.02)
        self.layer_id, self.seed, self.calls = int(layer_id) & 0xFF, int(seed), 0
        self._ws = None

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        if self._ws is None or self._ws.device != x.device:
            self._ws = binding.alloc_workspace(x.device)
        self.calls += 1
        tid = ((self.calls & 0xFFFFFF) << 8) | self.layer_id
        return fp4_linear(x, self.weight, seed=self.seed, tensor_id=tid, ws=self._ws)
