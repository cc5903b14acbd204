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
