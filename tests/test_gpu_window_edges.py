"""Windowed attention on the GPU at its edges: lengths far past a ring, layouts that leave the
matrix-core path, large launches of strided tensors, gradients of large scores."""
import pytest
import torch

from tests.test_gpu_window import BF16, DTYPES, run
from tests.window_reference import attention, visible

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


@DTYPES
def test_many_sequences_on_long_caches(dtype):
    """256 sequences of 8 key/value heads with caches of 131,072 tokens (one cache, seen from all)."""
    import paper_2604_16429_amd as M
    from paper_2604_16429_amd import binding
    B, h, kv, nk, D, left = 256, 16, 8, 131072, 64, 299
    gen = torch.Generator().manual_seed(11)
    k, v = (torch.randn(1, 1, nk, D, generator=gen).to(dtype).cuda() for _ in range(2))
    q = torch.randn(B, h, 1, D, generator=gen).to(dtype)
    lens = [1 + (i * 7919) % nk for i in range(B - 1)] + [nk]
    p = M.WindowParams(B, h, 1, nk, D, binding.BF16 if dtype is BF16 else binding.F32, kv_heads=kv,
                       window_left=left, n_sink=3)
    ws = torch.empty(max(256, M.mosaic_bsa_window_workspace_bytes(p, binding.OP_FWD)), dtype=torch.uint8,
                     device="cuda")
    out = torch.full((B, h, 1, D), float("nan"), dtype=dtype, device="cuda")
    M.mosaic_bsa_window_fwd(p, q.cuda(), k.expand(B, kv, -1, -1), v.expand(B, kv, -1, -1), out, workspace=ws,
                            k_lens=torch.tensor(lens, dtype=torch.int32).cuda())
    out, k, v = out.cpu().double(), k.cpu().double(), v.cpu().double()
    for b, n in enumerate(lens):
        rows = [j for j in range(3) if j < n - left - 1] + list(range(max(0, n - left - 1), n))
        see = torch.ones(1, len(rows), dtype=torch.bool)
        for i in range(0, h, 5):
            r = attention(q[b, i].double(), k[0, 0, rows], v[0, 0, rows], see, D ** -0.5)
            assert bool(((out[b, i] - r["out"]).abs() <= r["out_tol"](dtype)).all()), (b, i)


def test_training_of_many_long_slices():
    """1,024 slices of 262,177 tokens with the same queries, keys, values and upstream gradients: results of
    all are those of a call that has one of them."""
    import paper_2604_16429_amd as M
    from paper_2604_16429_amd import binding
    n, D, left, sinks = 262177, 32, 31, 2
    gen = torch.Generator().manual_seed(12)
    q, k, v, do = (torch.randn(1, 1, n, D, generator=gen).to(BF16).cuda() for _ in range(4))

    def train(B, h):
        p = M.WindowParams(B, h, n, n, D, binding.BF16, window_left=left, n_sink=sinks)

        def space(op):
            return torch.empty(max(256, M.mosaic_bsa_window_workspace_bytes(p, op)), dtype=torch.uint8,
                               device="cuda")

        a = [t.expand(B, h, n, D) for t in (q, k, v, do)]
        out, dq, dk, dv = (torch.full((B, h, n, D), float("nan"), dtype=BF16, device="cuda") for _ in range(4))
        lse = torch.full((B, h, n), float("nan"), device="cuda")
        M.mosaic_bsa_window_fwd(p, *a[:3], out, lse, workspace=space(binding.OP_FWD))
        M.mosaic_bsa_window_bwd(p, *a[:3], out, lse, a[3], dq, dk, dv, space(binding.OP_BWD))
        return out, dq, dk, dv

    one, all_ = train(1, 1), train(128, 8)
    for name, x, y in zip(("out", "dq", "dk", "dv"), one, all_):
        # (the queries beyond the window of the sinks are summed in another number of chunks)
        first = 32 if name in ("dk", "dv") else 0
        for b in range(128):
            assert bool((y[b] == y[0, :1]).all()), (name, b)
        assert torch.equal(x[0, 0, first:], y[0, 0, first:]), name
        assert bool(torch.isfinite(y[0, 0]).all())
    see = visible(300, 300, 300, 300, left, 0, sinks)
    x = [t[0, 0, :300].cpu().double() for t in (q, k, v)]
    r = attention(*x, see, D ** -0.5)
    assert bool(((one[0][0, 0, :300].cpu().double() - r["out"]).abs() <= r["out_tol"](BF16)).all())
    del one, all_, x, y
    torch.cuda.empty_cache()                       # (75 GB)


@DTYPES
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("left,right,sinks", [(63, -1, 0), (10, 900, 4), (300, 700, 33)])
def test_few_rows_with_keys_to_the_right(dtype, D, left, right, sinks):
    """Forward and backward of launches whose keys are shared out on both sides of a tile."""
    run(dtype, 1, 2, 1, 1500, 1500, D, left, right, sinks, train=True, seed=D + left)
    run(dtype, 2, 1, 1, 40, 1300, D, left, right, sinks, k_lens=[1300, 900], q_lens=[40, 33], seed=D)
