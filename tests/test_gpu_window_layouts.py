"""Windowed attention's training passes on the GPU: large launches of strided tensors, tensors whose rows
lie too far apart for the matrix-core kernels, large scores, scales of the caller's; bounds that count
each rounding once (window_bounds)."""
import pytest
import torch

from tests.test_gpu_window import BF16, DTYPES, FP32, run
from tests.window_bounds import check_training
from tests.window_reference import visible

pytestmark = pytest.mark.gpu


def heads_first(B, h, N, D):
    return h * N * D, N * D, D


def tokens_first(B, h, N, D):
    return N * h * D, D, h * D


def beside_others(B, h, N, D):
    """Parts of rows with 5 heads more."""
    return N * (h + 5) * D, D, (h + 5) * D


def rows_apart(stride):
    """Token rows `stride` elements apart, each with all batch entries and heads."""
    return lambda B, h, N, D: (h * D, D, stride)


def place(x, layout):
    """x [B, h, N, D] on the GPU with the strides of `layout`; what lies between is not initialised."""
    B, h, N, D = x.shape
    strides = (*layout(B, h, N, D), 1)
    size = 1 + sum((n - 1) * s for n, s in zip(x.shape, strides))
    t = torch.empty(size, dtype=x.dtype, device="cuda").as_strided(x.shape, strides)
    return t.copy_(x)


def train(B, h, kv, n, D, left, right, sinks, layouts, seed=0, q_lens=None, k_lens=None, scale=0.0,
          amplitude=1.0):
    """A training pass in bf16 with q, k, v, dout (and the results likewise) laid out by `layouts`."""
    import paper_2604_16429_amd as M
    from paper_2604_16429_amd import binding
    gen = torch.Generator().manual_seed(seed)
    q, k, v, g = (torch.randn(B, x, n, D, generator=gen) for x in (h, kv, kv, h))
    q, k, v, g = (q * amplitude).to(BF16), k.to(BF16), v.to(BF16), g.to(BF16)
    lay = dict(zip("qkvg", layouts))
    qd, kd, vd, gd = (place(x, lay[name]) for x, name in zip((q, k, v, g), "qkvg"))
    p = M.WindowParams(B, h, n, n, D, binding.BF16, kv_heads=kv, window_left=left, window_right=right,
                       n_sink=sinks, softmax_scale=scale)
    ql, kl = q_lens or [n] * B, k_lens or [n] * B
    lens = {name: torch.tensor(x, dtype=torch.int32).cuda()
            for name, x in (("q_lens", q_lens), ("k_lens", k_lens)) if x is not None}

    def space(op):
        size = max(256, M.mosaic_bsa_window_workspace_bytes(p, op))
        return torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")

    nan = torch.full_like(q, float("nan"))
    out, dq = place(nan, lay["g"]), place(nan, lay["q"])
    dk, dv = (place(torch.full_like(k, float("nan")), lay[name]) for name in "kv")
    lse = torch.full((B, h, n), float("nan"), device="cuda")
    M.mosaic_bsa_window_fwd(p, qd, kd, vd, out, lse, workspace=space(binding.OP_FWD), **lens)
    M.mosaic_bsa_window_bwd(p, qd, kd, vd, out, lse, gd, dq, dk, dv, space(binding.OP_BWD), **lens)
    for t, x in ((qd, q), (kd, k), (vd, v), (gd, g)):
        assert torch.equal(t.cpu(), x)             # inputs as they were
    got = {name: t.cpu().double() for name, t in
           (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv))}
    worst = check_training(got, *(x.double() for x in (q, k, v, g)), kv,
                           lambda b: visible(ql[b], kl[b], n, n, left, right, sinks), scale)
    print("share of the bound:", {name: round(x, 3) for name, x in worst.items()})


def ragged(B, n):
    return dict(q_lens=[n - (i * 37) % n if i % 3 else n for i in range(B)],
                k_lens=[n - (i * 23) % (n - 30) if i % 2 else n for i in range(B)])


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("left,right,sinks", [(15, 0, 2), (100, 0, 40), (30, 50, 0), (-1, 0, 0), (3, -1, 4)])
def test_small_launches(D, left, right, sinks):
    train(1, 4, 2, 290, D, left, right, sinks, [heads_first] * 4, seed=D + sinks)
    train(3, 3, 1, 131, D, left, right, sinks, [tokens_first] * 4, seed=D + left, **ragged(3, 131))


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("layout", [tokens_first, beside_others])
@pytest.mark.parametrize("left,right,sinks", [(100, 0, 4), (70, 50, 33), (300, 0, 0)])
def test_large_launches_of_strided_tensors(D, layout, left, right, sinks):
    """Enough workgroups for 128 rows and 128 keys to each, on the matrix-core path as well."""
    train(33, 4, 2, 389, D, left, right, sinks, [layout] * 4, seed=D + left, **ragged(33, 389))


@DTYPES
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("memory", ["tokens", "packed"])
def test_shared_walks_of_strided_tensors(dtype, D, memory):
    """160 workgroups of 128 keys, whose walks are shared out."""
    run(dtype, 40, 4, 1, 389, 389, D, 150, 0, 3, memory=memory, train=True, seed=D,
        q_lens=[389 - (i * 41) % 389 if i % 3 == 1 else 389 for i in range(40)])


FAR_ROWS = rows_apart(1 << 24)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("which", ["q", "dout", "k", "v"])
def test_rows_too_far_apart_for_the_matrix_core_kernels(D, which):
    """Token rows 2^24 elements apart leave 32-bit offsets: the general kernels, 128 rows and 128 keys to a
    workgroup, with the workspace of a call that is asked for without strides.  100 keys of 2^30 elements
    together in all."""
    layouts = [tokens_first] * 4
    at = {"q": 0, "k": 1, "v": 2, "dout": 3}[which]
    n = 100
    layouts[at] = FAR_ROWS if which in ("q", "dout") else rows_apart((1 << 30) // n // 8 * 8 + 8)
    train(70, 8, 4, n, D, 40, 0, 3, layouts, seed=D + at, **ragged(70, n))
    train(70, 8, 4, n, D, 20, 20, 0, layouts, seed=D + at + 1)
    # few workgroups: 32 rows and 32 keys to each
    train(2, 4, 2, n, D, 40, 0, 3, layouts, seed=D + at + 2)


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("B", [1, 40])
@pytest.mark.parametrize("kw", [dict(amplitude=30.0), dict(scale=2.0), dict(scale=0.01),
                                dict(amplitude=30.0, scale=0.3)], ids=str)
def test_gradients_of_scores_of_any_size(D, B, kw):
    """Weights that are one key's alone, where dP and delta nearly cancel, and even ones."""
    train(B, 4, 2, 200, D, 64, 0, 4, [heads_first] * 4, seed=D + B, **kw)


@pytest.mark.parametrize("kw", [dict(amplitude=30.0), dict(scale=2.0), dict(scale=0.01)], ids=str)
@pytest.mark.parametrize("D", [32, 64, 128])
def test_gradients_of_scores_of_any_size_in_full_precision(D, kw):
    run(FP32, 1, 4, 2, 200, 200, D, 64, 0, 4, train=True, seed=D, **kw)
    run(FP32, 40, 4, 2, 200, 200, D, 64, 0, 4, train=True, seed=D, **kw)
