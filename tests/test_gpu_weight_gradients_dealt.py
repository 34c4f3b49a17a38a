"""Weight gradients whose tiles are dealt: a call's counts are its own, whatever else uses its workspace."""
import numpy as np
import pytest
import torch

from paper_2607_24953_b200 import binding as b

pytestmark = pytest.mark.gpu


def skewed(T, e, seed):
    p = np.arange(1, e + 1) ** -0.8
    counts = np.random.RandomState(seed).multinomial(T, p / p.sum())
    return torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)).cuda()


def operands(seed, T, n, k):
    g = torch.Generator("cuda").manual_seed(seed)
    return [torch.randn(T, c, generator=g, device="cuda").to(torch.bfloat16) for c in (n, k)]


# pairs and single CTAs, with parts; the last without
SIZES = [(16384, 512, 1024, 40), (16384, 128, 640, 40), (5200, 1024, 512, 20), (2048, 4096, 2048, 8)]


@pytest.mark.parametrize("T,n,k,e", SIZES)
def test_what_lies_in_a_workspace_behind_its_settings_changes_nothing(T, n, k, e):
    dy, x = operands(1, T, n, k)
    offs = skewed(T, e, 2)
    spans = list(zip(offs[:-1].tolist(), offs[1:].tolist()))
    s = torch.cat([dy[i:j].double().abs().T @ x[i:j].double().abs() for i, j in spans])
    want = torch.cat([dy[i:j].double().T @ x[i:j].double() for i, j in spans])
    scratch = b.alloc_ragged_wgrad_scratch(T, n, k, e, "cuda")
    assert (scratch.numel() > 0) == (e > 8)
    ws = b.alloc_workspace("cuda")
    clean = b.fp4q_ragged_gemm_wgrad(dy, x, offs, ws=ws)
    # 32 instructions of 16 products a partial sum, 2^-22 each; a rounding for every partial sum of 512 elements
    longest = max(j - i for i, j in spans)
    assert ((clean.double() - want).abs() <= s * (32 * 2 ** -22 + (longest // 512 + 2) * 2 ** -24)).all()
    ws[16:] = 1                                              # as other calls that use it would leave it, or have it while they run
    kept = ws[16:].clone()
    for _ in range(3):
        scratch.fill_(255)
        assert torch.equal(b.fp4q_ragged_gemm_wgrad(dy, x, offs, ws=ws, scratch=scratch), clean)
    assert torch.equal(ws[16:], kept) and b.fp4q_workspace_status(ws) == 0


@pytest.mark.parametrize("shared", [True, False])
def test_two_streams_at_a_time(shared):
    # a workspace for both, which holds no more than the status, or one each; scratch memory is each call's own
    T, n, k, e = 16384, 512, 1024, 40
    jobs = [operands(i, T, n, k) + [skewed(T, e, i)] for i in (1, 2)]
    ws = [b.alloc_workspace("cuda")] * 2 if shared else [b.alloc_workspace("cuda") for _ in jobs]
    scratch = [b.alloc_ragged_wgrad_scratch(T, n, k, e, "cuda") for _ in jobs]
    want = [b.fp4q_ragged_gemm_wgrad(dy, x, offs, ws=ws[0]).clone() for dy, x, offs in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    outs = [[torch.full_like(w, 7.0) for _ in range(8)] for w in want]
    torch.cuda.synchronize()
    for r in range(8):
        for i, (dy, x, offs) in enumerate(jobs):
            b.fp4q_ragged_gemm_wgrad(dy, x, offs, out=outs[i][r], ws=ws[i], scratch=scratch[i], stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in (0, 1) for o in outs[i])
    assert all(b.fp4q_workspace_status(w) == 0 for w in ws)


def test_two_captured_graphs_with_one_workspace():
    T, n, k, e = 16384, 512, 1024, 40
    jobs = [operands(i, T, n, k) + [skewed(T, e, i)] for i in (3, 4)]
    ws = b.alloc_workspace("cuda")
    want = [b.fp4q_ragged_gemm_wgrad(dy, x, offs, ws=ws).clone() for dy, x, offs in jobs]
    torch.cuda.synchronize()
    graphs, got = [], []
    for dy, x, offs in jobs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(b.fp4q_ragged_gemm_wgrad(dy, x, offs, ws=ws))
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(8):
        for g in got:
            g.fill_(7.0)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))


def test_without_scratch_memory_they_go_in_turn():
    # The C entry's NULL: the same tiles, without parts.
    T, n, k, e = 5200, 1024, 512, 20
    dy, x = operands(1, T, n, k)
    offs, ws = skewed(T, e, 2), b.alloc_workspace("cuda")
    spans = list(zip(offs[:-1].tolist(), offs[1:].tolist()))
    out = torch.full((e * n, k), 7.0, device="cuda")
    import ctypes
    g = b._CGroups(e, 1, offs.data_ptr())
    stream = torch.cuda.current_stream().cuda_stream
    assert b.lib().fp4q_ragged_gemm_wgrad(dy.data_ptr(), T, n, n, x.data_ptr(), k, k, out.data_ptr(), k, b.OUT_F32, 0, ctypes.byref(g), None, 0, ws.data_ptr(),
                                          ws.numel(), stream) == 0
    want = torch.cat([dy[i:j].double().T @ x[i:j].double() for i, j in spans])
    s = torch.cat([dy[i:j].double().abs().T @ x[i:j].double().abs() for i, j in spans])
    assert ((out.double() - want).abs() <= s * (32 * 2 ** -22 + (max(j - i for i, j in spans) // 512 + 2) * 2 ** -24)).all()


def test_many_rows_do_not_add_up_what_bf16_accumulators_cut_off():
    # Sums of one sign over 2^20 rows.  An accumulator takes 131072 of them at most, in 8192 instructions that cut off less than 2^-22 of a sum that grows
    # evenly: 4096 * 2^-22 = 9.8e-4 of the result.  Rounding to BF16 is right in the mean: 2^-8 / sqrt(3) / sqrt(32768) for the columns' several sizes.
    T, n, k = 1 << 20, 768, 2048
    g = torch.Generator("cuda").manual_seed(1)
    dy = torch.rand(T, n, generator=g, device="cuda").to(torch.bfloat16)
    x = (torch.rand(T, k, generator=g, device="cuda") * (1 + torch.rand(k, generator=g, device="cuda"))).to(torch.bfloat16)
    got = b.fp4q_ragged_gemm_wgrad(dy, x, dt=b.OUT_BF16)[:64, :512].double()
    want = dy[:, :64].double().T @ x[:, :512].double()
    off = (got - want) / want
    assert off.mean().abs() <= 4096 * 2 ** -22 + 5 * 2 ** -8 / 3 ** 0.5 / 32768 ** 0.5 and off.abs().max() <= 4096 * 2 ** -22 + 2 ** -8
