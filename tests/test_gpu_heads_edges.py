"""Rotation and head norms on the GPU at their edges: no epsilon, far positions, gradients over
their inputs."""
import pytest
import torch

from tests.test_gpu_heads import (BF16, DTYPES, FP32, U32, check, frequencies, lib, nan_like, normed,
                                  pair_size, rotation_tol, tensor)
from tests.test_rotation_angles import TWO_PI, decimal_frequencies, fraction
from tests.window_reference import HALF_STEP, rotate

pytestmark = pytest.mark.gpu


@DTYPES
@pytest.mark.parametrize("D,rd", [(32, 32), (64, 24), (128, 128)])
@pytest.mark.parametrize("N", [1, 33, 70])
def test_norm_gradients_without_an_epsilon(dtype, D, rd, N):
    """norm_eps 0, and token counts that leave lanes of the last workgroup without a row."""
    M, binding = lib()
    B, h, kv = 1, 3, 1
    gen = torch.Generator().manual_seed(D + N)
    q, q64 = tensor((B, h, N, D), dtype, gen, "tokens")
    k, k64 = tensor((B, kv, N, D), dtype, gen, "tokens")
    gq, gq64 = tensor((B, h, N, D), dtype, gen, "heads")
    gk, gk64 = tensor((B, kv, N, D), dtype, gen, "heads")
    qw, kw = (1.0 + 0.3 * torch.randn(D, generator=gen) for _ in range(2))
    p = M.HeadsParams(B, N, h, D, binding.BF16 if dtype is BF16 else binding.F32, kv_heads=kv,
                      norm_eps=0.0)
    rot = M.Rotation(rd)
    dq, dk = nan_like(q), nan_like(k)
    dqw, dkw = (torch.full((D,), float("nan"), device="cuda") for _ in range(2))
    ws = torch.full((M.mosaic_bsa_qk_norm_rope_workspace_bytes(p),), 0xff, dtype=torch.uint8,
                    device="cuda")
    M.mosaic_bsa_qk_norm_rope_bwd(p, rot, None, q, k, qw.cuda(), kw.cuda(), gq, gk, dq, dk, dqw, dkw,
                                  ws)
    pos = torch.arange(N).view(1, N, 1)
    for x64, w, g64, dx, dw, name in ((q64, qw, gq64, dq, dqw, "q"), (k64, kw, gk64, dk, dkw, "k")):
        x = x64.clone().requires_grad_(True)
        w = w.double().requires_grad_(True)
        y = rotate(normed(x, w, 0.0), pos, frequencies(rd), 1.0, rd, 1, False)
        rx, rw = torch.autograd.grad(y, (x, w), g64)
        # the norm: a sum of D squares, a root and a quotient: (D / 2 + 6) roundings of 2^-24;
        # dx = r (dn - n mean(dn n)): bounds of its two terms, each good to 2 rel + rotation
        rel = (D / 2 + 6) * U32
        r = 1.0 / torch.sqrt((x64 * x64).mean(-1, keepdim=True))
        dn, n = pair_size(g64) * w.detach().abs(), (x64 * r).abs()
        size = r * (dn + n * (dn * n).mean(-1, keepdim=True))
        check(dx, rx, size * (4 * rel + 16 * U32) + rx.abs() * HALF_STEP[dtype], "d" + name)
        # dw: at most a few dozen values to a lane in 32 bits, then 64
        total = (pair_size(g64) * n).sum((0, 1, 2))
        check(dw, rw, total * (2 * rel + 16 * U32) + rw.abs() * U32, "d" + name + "_weight")


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("first", [0, -2 ** 31, 2 ** 31 - 40, 2 ** 30 + 12345])
def test_far_positions_against_exact_angles(first, transpose):
    """Angles of the reference in decimal arithmetic: no allowance beside the kernel's own."""
    M, binding = lib()
    N, D = 40, 64
    gen = torch.Generator().manual_seed(2)
    q, q64 = tensor((1, 1, N, D), FP32, gen, "heads")
    pos = torch.arange(N) + first
    out = nan_like(q)
    p = M.HeadsParams(1, N, 1, D, binding.F32)
    (M.mosaic_bsa_rope_bwd if transpose else M.mosaic_bsa_rope_fwd)(
        p, M.Rotation(D), pos.to(torch.int32).cuda(), q, None, out, None)
    angle = torch.tensor([[float(fraction(int(x) * w / TWO_PI) * TWO_PI) for w in decimal_frequencies(D)]
                          for x in pos], dtype=torch.float64)
    c, s = torch.cos(angle), torch.sin(angle) * (-1.0 if transpose else 1.0)
    a, b = q64[0, 0].chunk(2, -1)
    ref = torch.cat([a * c - b * s, b * c + a * s], -1).view(1, 1, N, D)
    check(out, ref, rotation_tol(ref, pair_size(q64), FP32), "q")


@DTYPES
@pytest.mark.parametrize("D,rd,memory", [(32, 32, "tokens"), (64, 24, "heads"), (128, 128, "tokens"), (64, 62, 3)])
def test_norm_gradients_over_their_inputs(dtype, D, rd, memory):
    """dq and dk may be q and k: the same bits as in memory of their own."""
    M, binding = lib()
    B, h, kv, N = 2, 5, 2, 70
    gen = torch.Generator().manual_seed(D)
    q, k = (tensor((B, x, N, D), dtype, gen, memory)[0] for x in (h, kv))
    gq, gk = (tensor((B, x, N, D), dtype, gen, "heads")[0] for x in (h, kv))
    qw, kw = (1.0 + 0.3 * torch.randn(D, generator=gen).cuda() for _ in range(2))
    p = M.HeadsParams(B, N, h, D, binding.BF16 if dtype is BF16 else binding.F32, kv_heads=kv)
    rot = M.Rotation(rd)
    ws = torch.empty(M.mosaic_bsa_qk_norm_rope_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    results = []
    for over in (False, True):
        dq, dk = (q, k) if over else (nan_like(q), nan_like(k))
        dw = torch.full((2, D), float("nan"), device="cuda")
        M.mosaic_bsa_qk_norm_rope_bwd(p, rot, None, q, k, qw, kw, gq, gk, dq, dk, dw[0], dw[1], ws)
        results.append([t.clone() for t in (dq, dk, dw)])
    for a, b in zip(*results):
        assert bool(torch.isfinite(a).all()) and torch.equal(a, b)


@DTYPES
def test_rotated_heads_go_into_the_selection(dtype, oracle):
    """Queries and keys rotated by their grid positions, then block selection and attention on them, against
    the oracle on the rotated values."""
    import dataclasses

    from inputs.fields import make_problem, round_to_bf16
    from tests import gpu_util
    M, binding = lib()
    prob = make_problem(1)
    cfg = dataclasses.replace(prob.cfg, dtype="bf16" if dtype is BF16 else "fp32")
    q, k, v = (round_to_bf16(x) if dtype is BF16 else x for x in (prob.q, prob.k, prob.v))
    qd, kd = gpu_util.to_dev(q, cfg), gpu_util.to_dev(k, cfg)
    N = cfg.grid_h * cfg.grid_w
    t = torch.arange(N, dtype=torch.int32)
    pos = torch.stack([t // cfg.grid_w, t % cfg.grid_w], -1)
    qr, kr = torch.full_like(qd, float("nan")), torch.full_like(kd, float("nan"))
    M.mosaic_bsa_rope_fwd(
        M.HeadsParams(cfg.batch, N, cfg.heads, cfg.head_dim, binding.BF16 if dtype is BF16 else binding.F32,
                      kv_heads=kd.shape[1]),
        M.Rotation(cfg.head_dim, axes=2), pos.cuda(), qd, kd, qr, kr)
    for got, x in ((qr, qd), (kr, kd)):
        x64 = x.cpu().double()
        ref = rotate(x64, pos.unsqueeze(0), frequencies(cfg.head_dim // 2), 1.0, cfg.head_dim, 2, False)
        check(got, ref, rotation_tol(ref, pair_size(x64), dtype), "rotated")
    idx = gpu_util.select_dev(cfg, qr, kr)
    out, _ = gpu_util.fwd_dev(cfg, qr, kr, gpu_util.to_dev(v, cfg), idx)
    rotated = [x.float().cpu().numpy() for x in (qr, kr)]
    s = oracle.shape_of(cfg)
    want = oracle.select(s, *rotated)
    assert (idx.cpu().numpy() == want).all()
    ref, _ = oracle.fwd(s, *rotated, v, want)
    off = abs(out.float().cpu().numpy() - ref).max()
    # bf16: a weight's and the result's rounding, 2^-8 each of the largest value; fp32: as elsewhere
    assert off <= (2.0 ** -7 if dtype is BF16 else 1e-5) * abs(v).max()


def test_given_frequencies_with_a_magnitude():
    M, binding = lib()
    N, D = 50, 64
    gen = torch.Generator().manual_seed(8)
    q, q64 = tensor((1, 2, N, D), FP32, gen, "heads")
    freq = [0.5 / (1 + i) for i in range(D // 2)]
    rot = M.Rotation(D, inv_freq=freq)
    assert rot.c.magnitude == 1.0
    rot.c.magnitude = 1.25
    out = nan_like(q)
    M.mosaic_bsa_rope_fwd(M.HeadsParams(1, N, 2, D, binding.F32), rot, None, q, None, out, None)
    ref = rotate(q64, torch.arange(N).view(1, N, 1), freq, 1.25, D, 1, False)
    check(out, ref, rotation_tol(ref, pair_size(q64) * 1.25, FP32), "q")
