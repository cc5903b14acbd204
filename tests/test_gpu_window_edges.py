"""Windowed attention on the GPU at its edges: lengths far past a ring, layouts that leave the
matrix-core path, large launches of strided tensors, gradients of large scores."""
import pytest
import torch

from tests.test_gpu_window import BF16, DTYPES, FP32, run

pytestmark = pytest.mark.gpu


@DTYPES
@pytest.mark.parametrize("D,nq,right", [(64, 1, 0), (128, 5, 0), (32, 40, -1), (64, 1, -1)])
def test_rings_that_have_turned_for_long(dtype, D, nq, right):
    """A length counts modulo the ring: past 2^30, and up to the longest one, the same bits."""
    import paper_2604_16429_amd as M
    from paper_2604_16429_amd import binding
    sinks, ring, left = 4, 100, 59
    most = 3 << 29
    first = [sinks + 3 * ring + 7, sinks + 2 * ring, sinks + ring + 41, (most - sinks) % ring + 2 * ring + sinks]
    far = [first[0] + (1 << 30) // ring * ring, first[1] + 12_000_000 * ring, first[2], most]
    for a, b in zip(first, far):
        assert b <= most and (b - a) % ring == 0
    gen = torch.Generator().manual_seed(D + nq)
    q, k, v = (torch.randn(4, 2, n, D, generator=gen).to(dtype).cuda() for n in (nq, 104, 104))
    p = M.WindowParams(4, 2, nq, sinks + ring, D, binding.BF16 if dtype is BF16 else binding.F32,
                       window_left=left, window_right=right, n_sink=sinks, ring=ring)
    ws = torch.empty(max(256, M.mosaic_bsa_window_workspace_bytes(p, binding.OP_FWD)), dtype=torch.uint8,
                     device="cuda")
    outs = []
    for lens in (first, far):
        out = torch.full_like(q, float("nan"))
        lse = torch.full((4, 2, nq), float("nan"), device="cuda")
        M.mosaic_bsa_window_fwd(p, q, k, v, out, lse, workspace=ws,
                                k_lens=torch.tensor(lens, dtype=torch.int32).cuda())
        outs.append((out.cpu(), lse.cpu()))
    assert bool(torch.isfinite(outs[0][1]).all())
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
