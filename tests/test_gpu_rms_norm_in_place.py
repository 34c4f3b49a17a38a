"""The norm's gradient written over each of the matrices that it is computed from, at widths of every kernel: what is written elsewhere, bit for bit."""
import pytest
import torch

from paper_2607_24953_b200 import binding as b

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def pitched(t, ld):
    buf = torch.zeros(t.shape[0], ld, dtype=t.dtype, device="cuda")[:, :t.shape[1]]
    return buf.copy_(t)


@pytest.mark.parametrize("ty,th", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("rows,cols,pad", [(1, 40, 0), (600, 401, 0), (700, 4096, 8), (700, 8192, 0), (700, 8193, 3), (900, 9000, 0), (300, 16384, 16), (300, 16411, 0), (20, 40000, 0), (300, 65536, 0)])
def test_over_h_dy_and_dh(rows, cols, pad, ty, th):
    dy, h, dh = pitched(randn(1, rows, cols).to(ty), cols + pad), pitched(randn(2, rows, cols).to(th), cols + pad), pitched(randn(3, rows, cols).to(th), cols + pad)
    w, rstd = randn(4, cols), torch.rsqrt(h.float().square().mean(1) + 1e-6)
    want, dw = b.fp4q_rms_norm_bwd(dy, h, rstd, w, dh=dh)
    for over in ("h", "dh", "dy"):
        t = {"h": h, "dh": dh, "dy": dy}
        if t[over].dtype != th:
            continue
        t[over] = pitched(t[over], cols + pad)
        got, dw2 = b.fp4q_rms_norm_bwd(t["dy"], t["h"], rstd, w, dh=t["dh"], out=t[over])
        assert got is t[over] and torch.equal(got, want) and torch.equal(dw2, dw), over
