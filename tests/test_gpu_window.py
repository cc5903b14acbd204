"""Windowed attention with sinks on the GPU against the definition in 64 bits: forward,
single tokens, chunks, ring caches and gradients, at the sizes and masks where tiles, lengths
and layouts meet."""
import math

import pytest
import torch

from tests.window_reference import HALF_STEP, attention, visible

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def make(shape, memory, dtype, gen, heads_of):
    """A [B, h, N, D] tensor with the memory of `memory`, and its values on the CPU in 64 bits."""
    B, h, N, D = shape
    x = torch.randn(shape, generator=gen).to(dtype)
    if memory == "heads":
        t = x.cuda()
    elif memory == "tokens":
        t = x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    else:                             # a part of wider rows, with a gap on both sides
        wide = torch.full((B, N, heads_of + 2, D), float("nan"), dtype=dtype)
        wide[:, :, 1:1 + h] = x.transpose(1, 2)
        t = wide.cuda()[:, :, 1:1 + h].transpose(1, 2)
    return t, x.double()


def empty_like_memory(t):
    """A tensor of NaN with the strides of t in memory of its own."""
    out = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device)
    out.fill_(float("nan"))
    return out


def run(dtype, B, h, kv, nq, nk, D, left, right, sinks, q_lens=None, k_lens=None, memory="heads",
        ring=0, train=False, seed=0, scale=0.0, amplitude=1.0, junk=True):
    import paper_2604_16429_amd as M
    from paper_2604_16429_amd import binding
    gen = torch.Generator().manual_seed(1000 + seed)
    q, q64 = make((B, h, nq, D), memory, dtype, gen, h)
    k, k64 = make((B, kv, nk, D), memory, dtype, gen, kv)
    v, v64 = make((B, kv, nk, D), memory, dtype, gen, kv)
    if amplitude != 1.0:
        q.mul_(amplitude)
        q64 = q.cpu().double()
    ql = q_lens if q_lens is not None else [nq] * B
    kl = k_lens if k_lens is not None else [nk] * B
    if junk and not ring:
        # what no query sees may hold anything
        for b in range(B):
            unseen = ~visible(min(ql[b], nq), min(kl[b], nk), nq, nk, left, right, sinks).any(0)
            k[b, :, unseen.cuda()] = float("nan")
            v[b, :, unseen.cuda()] = float("inf")
            q[b, :, ql[b]:] = float("nan")
    p = M.WindowParams(B, h, nq, nk, D, binding.BF16 if dtype is BF16 else binding.F32, kv_heads=kv,
                       window_left=left, window_right=right, n_sink=sinks, ring=ring,
                       softmax_scale=scale)
    lens = dict(q_lens=None if q_lens is None else torch.tensor(q_lens, dtype=torch.int32).cuda(),
                k_lens=None if k_lens is None else torch.tensor(k_lens, dtype=torch.int32).cuda())
    n = M.mosaic_bsa_window_workspace_bytes(p, binding.OP_FWD)
    ws = torch.full((max(n, 256),), 0xff, dtype=torch.uint8, device="cuda")
    out = empty_like_memory(q)
    lse = torch.full((B, h, nq), float("nan"), device="cuda")
    M.mosaic_bsa_window_fwd(p, q, k, v, out, lse, workspace=ws, **lens)
    again = empty_like_memory(q)
    M.mosaic_bsa_window_fwd(p, q, k, v, again, None, workspace=ws, **lens)
    got = {"out": out, "lse": lse}
    assert torch.equal(out, again)                 # the same bits, with and without lse
    do64 = None
    if train:
        do, do64 = make((B, h, nq, D), memory, dtype, gen, h)
        for b in range(B):
            do[b, :, ql[b]:] = float("nan")
        got["dq"], got["dk"], got["dv"] = (empty_like_memory(t) for t in (q, k, v))
        n = M.mosaic_bsa_window_workspace_bytes(p, binding.OP_BWD)
        ws = torch.full((max(n, 256),), 0xff, dtype=torch.uint8, device="cuda")
        M.mosaic_bsa_window_bwd(p, q, k, v, out, lse, do, got["dq"], got["dk"], got["dv"], ws, **lens)
        second = [empty_like_memory(t) for t in (q, k, v)]
        M.mosaic_bsa_window_bwd(p, q, k, v, out, lse, do, *second, ws, **lens)
        for name, t in zip(("dq", "dk", "dv"), second):
            assert torch.equal(got[name], t), name
    torch.cuda.synchronize()
    got = {name: t.cpu().double() for name, t in got.items()}

    sc = scale if scale > 0.0 else 1.0 / math.sqrt(D)
    G = h // kv
    worst = {}

    def close(name, x, ref, tol):
        d = (x - ref).abs()
        same = x == ref                            # (-infinity of an empty row)
        bad = ~same & ~(d <= tol)
        ratio = float(torch.where(same, torch.zeros_like(d), d / tol).max())
        worst[name] = max(worst.get(name, 0.0), ratio)
        assert not bool(bad.any()), f"{name}: {int(bad.sum())} values off, worst {ratio} of the bound"

    for b in range(B):
        kvis = min(kl[b], nk) if not ring else kl[b]
        see = visible(min(ql[b], nq), kvis, nq, max(nk, kvis), left, right, sinks)
        for a in range(kv):
            if ring:
                j = torch.arange(see.shape[1])
                rows = torch.where(j < sinks, j, sinks + (j - sinks) % ring)
                kk, vv = k64[b, a][rows], v64[b, a][rows]
            else:
                kk, vv = k64[b, a], v64[b, a]
            sums = {}
            for i in range(a * G, (a + 1) * G):
                g = None if do64 is None else do64[b, i].masked_fill(
                    torch.arange(nq).unsqueeze(1) >= min(ql[b], nq), 0.0)
                qq = q64[b, i].masked_fill(torch.arange(nq).unsqueeze(1) >= min(ql[b], nq), 0.0)
                r = attention(qq, kk, vv, see, sc, g)
                close("out", got["out"][b, i], r["out"], r["out_tol"](dtype))
                close("lse", got["lse"][b, i], r["lse"], r["lse_tol"])
                if train:
                    close("dq", got["dq"][b, i], r["dq"],
                          r["dq_tol"](dtype) + r["dq"].abs() * HALF_STEP[dtype])
                    for name in ("dk", "dv"):
                        s = sums.setdefault(name, [0.0, 0.0])
                        s[0] = s[0] + r[name]
                        s[1] = s[1] + r[name + "_tol"](dtype)
            for name, (ref, tol) in sums.items():
                close(name, got[name][b, a], ref, tol + ref.abs() * HALF_STEP[dtype])
    print("share of the bound:", {n: round(x, 3) for n, x in worst.items()})
    return got


DTYPES = pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])


@DTYPES
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("h,kv", [(2, 2), (4, 1), (5, 1), (6, 2)])
def test_whole_sequences(dtype, D, h, kv):
    run(dtype, 2, h, kv, 197, 197, D, 40, 0, 3, train=True, seed=D + h)


@DTYPES
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300])
def test_lengths_around_the_tiles(dtype, n):
    run(dtype, 1, 2, 1, n, n, 64, 63, 0, 4, train=True, seed=n)


@DTYPES
@pytest.mark.parametrize("left,right,sinks", [
    (0, 0, 0), (0, 0, 1), (0, 0, 64), (1, 0, 0), (-1, 0, 0), (-1, 0, 7), (-1, -1, 0), (31, 31, 2),
    (16, -1, 5), (64, 3, 64), (200, 0, 129), (5, 100, 33), (1000, 1000, 1000), (15, 0, 140)])
def test_windows(dtype, left, right, sinks):
    run(dtype, 1, 4, 2, 290, 290, 64, left, right, sinks, train=True, seed=left + sinks + 2)


@DTYPES
@pytest.mark.parametrize("memory", ["tokens", "packed"])
def test_memory_layouts(dtype, memory):
    run(dtype, 2, 6, 2, 150, 150, 64, 50, 0, 4, memory=memory, train=True)
    run(dtype, 2, 6, 2, 9, 150, 128, 50, 0, 4, memory=memory)


@DTYPES
def test_sequences_of_their_own_lengths(dtype):
    """Lengths of 0 and 1, queries without keys, more queries than keys."""
    run(dtype, 7, 4, 2, 140, 140, 64, 30, 0, 4, q_lens=[140, 0, 1, 77, 100, 64, 5],
        k_lens=[140, 50, 1, 77, 30, 0, 139], train=True)
    run(dtype, 4, 3, 1, 70, 333, 32, 100, 2, 2, q_lens=[70, 1, 33, 64], k_lens=[333, 300, 20, 65],
        train=True)


@DTYPES
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("h,kv", [(1, 1), (4, 1), (8, 2), (20, 4), (40, 1)])
def test_single_tokens(dtype, D, h, kv):
    run(dtype, 3, h, kv, 1, 700, D, 511, 0, 4, k_lens=[700, 1, 513], q_lens=[1, 1, 1])


@DTYPES
@pytest.mark.parametrize("nk,left,sinks", [(1, 0, 0), (17, -1, 0), (64, 63, 0), (65, 63, 1),
                                           (1025, 1023, 2), (3001, -1, 0), (3001, 2047, 5)])
@pytest.mark.parametrize("nq", [1, 3, 17])
def test_few_tokens_on_caches(dtype, nk, left, sinks, nq):
    nq = min(nq, nk)
    run(dtype, 2, 4, 2, nq, nk, 64, left, 0, sinks, k_lens=[nk, max(nq, nk // 2)], q_lens=[nq, nq])


@DTYPES
@pytest.mark.parametrize("nq", [1, 5])
@pytest.mark.parametrize("sinks,ring", [(0, 128), (4, 128), (3, 77), (64, 300)])
def test_ring_caches(dtype, nq, sinks, ring):
    left = ring - nq - (ring % 3)
    run(dtype, 4, 4, 2, nq, sinks + ring, 64, left, 0, sinks, ring=ring,
        k_lens=[nq, ring + sinks, ring + sinks + 1, 3 * ring + 5], q_lens=[nq, 1, nq, nq])


@DTYPES
def test_scores_of_any_size(dtype):
    """Weights that are one key's alone, and sums that move the reference."""
    run(dtype, 1, 2, 1, 200, 200, 64, 64, 0, 4, amplitude=30.0, seed=7)
    run(dtype, 1, 2, 1, 1, 2000, 64, 1500, 0, 4, amplitude=30.0, seed=8)
    run(dtype, 1, 2, 1, 130, 130, 64, 64, 0, 4, scale=2.0, seed=9)


def test_gradients_against_differences():
    """dq, dk, dv against central differences of the 64-bit forward along random directions."""
    D, n, left, sinks = 32, 90, 20, 3
    got = run(FP32, 1, 2, 1, n, n, D, left, 0, sinks, train=True, seed=77)
    gen = torch.Generator().manual_seed(1077)
    q, k, v = (torch.randn(1, x, n, D, generator=gen).double() for x in (2, 1, 1))
    do = torch.randn(1, 2, n, D, generator=gen).double()
    see = visible(n, n, n, n, left, 0, sinks)

    def loss(q, k, v):
        total = 0.0
        for i in range(2):
            r = attention(q[0, i], k[0, 0], v[0, 0], see, 1.0 / math.sqrt(D))
            total += float((r["out"] * do[0, i]).sum())
        return total

    gen = torch.Generator().manual_seed(5)
    for name, at in (("dq", 0), ("dk", 1), ("dv", 2)):
        x = [q, k, v]
        d = torch.randn(x[at].shape, generator=gen).double()
        h = 1e-5
        x[at] = x[at] + h * d
        up = loss(*x)
        x[at] = x[at] - 2 * h * d
        down = loss(*x)
        want = (up - down) / (2 * h)
        have = float((got[name] * d).sum())
        # rounding of the gradients in 32 bits, and h^2 of the differences
        assert abs(have - want) <= 1e-4 * float(d.norm() * got[name].norm())


def test_rows_far_into_a_long_cache():
    """Offsets past 2^32 bytes: one sequence of 2^24 + 1,000 tokens at head dim 128."""
    import paper_2604_16429_amd as M
    from paper_2604_16429_amd import binding
    n, D, left = (1 << 24) + 1000, 128, 299
    cache = torch.zeros(2, 1, 1, n, D, dtype=BF16, device="cuda")
    gen = torch.Generator().manual_seed(3)
    tail = torch.randn(2, 400, D, generator=gen).to(BF16)
    cache[:, 0, 0, -400:] = tail.cuda()
    for nq in (1, 40, 300):
        q = torch.randn(1, 2, nq, D, generator=gen).to(BF16)
        p = M.WindowParams(1, 2, nq, n, D, binding.BF16, kv_heads=1, window_left=left)
        ws = torch.empty(max(256, M.mosaic_bsa_window_workspace_bytes(p, binding.OP_FWD)),
                         dtype=torch.uint8, device="cuda")
        out = torch.full((1, 2, nq, D), float("nan"), dtype=BF16, device="cuda")
        M.mosaic_bsa_window_fwd(p, q.cuda(), cache[0], cache[1], out, workspace=ws)
        keys = min(400, left + nq)
        # keys before the last 400 are zeros
        k64 = torch.zeros(left + nq, D).double()
        v64 = torch.zeros(left + nq, D).double()
        k64[-keys:], v64[-keys:] = tail[0, -keys:].double(), tail[1, -keys:].double()
        see = visible(nq, left + nq, nq, left + nq, left, 0, 0)
        for i in range(2):
            r = attention(q[0, i].double(), k64, v64, see, 1.0 / math.sqrt(D))
            d = (out[0, i].cpu().double() - r["out"]).abs()
            assert bool((d <= r["out_tol"](BF16)).all())


@DTYPES
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("h,kv,left,right,sinks", [(4, 1, 100, 0, 4), (3, 1, 70, 50, 33), (1, 1, 300, 0, 200)])
def test_many_key_tiles(dtype, D, h, kv, left, right, sinks):
    """Batches that fill the chip: 128 keys to a workgroup in the backward."""
    n = 389
    B = 64 // kv + 1
    run(dtype, B, h, kv, n, n, D, left, right, sinks, train=True, seed=D + left,
        q_lens=[n - (i * 37) % n if i % 3 else n for i in range(B)],
        k_lens=[n - (i * 23) % 350 if i % 2 else n for i in range(B)])


@DTYPES
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("B,h,n,left,right,sinks", [
    (1, 5, 300, -1, 0, 0), (1, 5, 300, 250, 0, 40),         # 32 keys a workgroup
    (40, 4, 389, 150, 0, 3), (40, 4, 389, -1, -1, 0),       # 160 workgroups of 128
    (60, 4, 520, 500, 500, 2)])                             # 300
def test_shared_walks(dtype, D, B, h, n, left, right, sinks):
    """Backward launches in which several workgroups have the same keys."""
    run(dtype, B, h, 1, n, n, D, left, right, sinks, train=True, seed=D + n,
        q_lens=[n - (i * 41) % n if i % 3 == 1 else n for i in range(B)],
        k_lens=[n - (i * 29) % 300 if i % 2 else n for i in range(B)])


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("B,n", [(1, 400), (24, 600)])
def test_roundings_of_bf16_gradients(D, B, n):
    """dQ and dK carry two independent roundings, that of dS and that of the result: sqrt(2) times the
    latter's error in the 2-norm, and no more than 1.5 times with what else there is.  Short windows,
    where delta out of the rounded output would add as much again."""
    h, kv, left, right, sinks = 4, 2, 15, 0, 2
    got = run(BF16, B, h, kv, n, n, D, left, right, sinks, train=True, seed=D + n, junk=False)
    gen = torch.Generator().manual_seed(1000 + D + n)
    q, k, v = (torch.randn(B, x, n, D, generator=gen).to(BF16).double() for x in (h, kv, kv))
    do = torch.randn(B, h, n, D, generator=gen).to(BF16).double()
    see = visible(n, n, n, n, left, right, sinks)
    want = {"dq": torch.zeros_like(q), "dk": torch.zeros_like(k)}
    for b in range(B):
        for i in range(h):
            r = attention(q[b, i], k[b, i // 2], v[b, i // 2], see, 1.0 / math.sqrt(D), do[b, i])
            want["dq"][b, i] = r["dq"]
            want["dk"][b, i // 2] += r["dk"]
    for name, w in want.items():
        rounding = float((w.to(BF16).double() - w).norm())
        assert float((got[name] - w).norm()) <= 1.5 * rounding, name
