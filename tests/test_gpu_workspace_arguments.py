"""Workspaces and scratch memory that a kernel could not write to are refused before anything is launched."""
import pytest
import torch

from paper_2607_24953_b200 import autograd, binding as b

pytestmark = pytest.mark.gpu


def test_of_another_device_or_with_gaps():
    x, w = torch.zeros(64, 32, dtype=torch.bfloat16, device="cuda"), torch.zeros(96, 32, dtype=torch.bfloat16, device="cuda")
    g, offs = torch.zeros(40, 50, device="cuda"), torch.tensor([0, 30, 64], device="cuda")
    dy = torch.zeros(64, 48, dtype=torch.bfloat16, device="cuda")
    qx, qw = b.fp4q_quantize2d(x), b.fp4q_quantize2d(w)
    for bad in (torch.zeros(256, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8, device="cuda")[::2], torch.zeros(1, dtype=torch.uint8, device="cuda").expand(256)):
        for call in (lambda: b.fp4q_ragged_gemm_fwd(x, w, offs, ws=bad), lambda: b.fp4q_ragged_gemm_dgrad(dy, w, offs, ws=bad),
                     lambda: b.fp4q_ragged_gemm_wgrad(dy, x, offs, ws=bad), lambda: b.fp4q_newton_schulz(g, ws=bad), lambda: b.fp4q_gemm_fwd(qx, qw, ws=bad),
                     lambda: autograd.ragged_linear(x, w.view(2, 48, 32), offs, ws=bad), lambda: b.fp4q_newton_schulz(g, scratch=bad),
                     lambda: b.fp4q_ragged_gemm_wgrad(dy, x, offs, scratch=bad)):
            with pytest.raises(ValueError, match="ws must|scratch must"):
                call()
    ws = b.alloc_workspace("cuda")
    assert not b.fp4q_ragged_gemm_fwd(x, w, offs, ws=ws).any() and not b.fp4q_newton_schulz(g, ws=ws).any() and not b.fp4q_gemm_fwd(qx, qw, ws=ws).any()
    assert b.fp4q_workspace_status(ws) == 0
