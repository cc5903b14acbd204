"""New tokens into a cache in pages on the GPU: against the definition in 64 bits and against the entry points
for contiguous caches, with every row that is no new token's left as it was."""
import math

import pytest
import torch

from tests.paged_reference import BF16, FP32, strided
from tests.window_reference import HALF_STEP, rotate

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])
U32 = 2.0 ** -24


def lib():
    import paper_2604_16429_amd as M
    from paper_2604_16429_amd import binding
    return M, binding


def same_bits(a, b):
    kind = {2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


def normed(x, w, eps):
    return w.double() * x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)


def run(dtype, B, h, kv, N, D, T, q_lens, k_lens, width, prefix=0, prefix_len=None, rd=None, axes=1,
        pairs=False, norm=False, positions=None, memory="heads", order="heads", bad=(), in_place=False,
        seed=0):
    M, binding = lib()
    gen = torch.Generator().manual_seed(3000 + seed)
    rd = D if rd is None else rd
    new = {n: torch.randn(B, c, N, D, generator=gen).to(dtype) for n, c in (("q", h), ("k", kv), ("v", kv))}
    ql = [N] * B if q_lens is None else [min(max(x, 0), N) for x in q_lens]
    kl = [min(max(x, 0), width * T) for x in k_lens]
    dev = {n: strided(x, memory) for n, x in new.items()}
    pages = B * width + 3
    table = torch.randperm(pages, generator=gen)[:B * width].view(B, width).to(torch.int32)
    named = table.clone()
    for x, (b, i) in enumerate(bad):
        table[b, i] = (-1, pages, -(2 ** 31), 2 ** 31 - 1)[x % 4]
    shape = (pages, kv, T, D)
    pools = {n: torch.randn(shape, generator=gen).to(dtype) for n in ("k", "v")}
    if order == "tokens":
        pool = {n: x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for n, x in pools.items()}
    else:
        pool = {n: x.cuda() for n, x in pools.items()}
    P = prefix if prefix_len is None else min(max(prefix_len, 0), prefix)
    wq, wk = ((1.0 + 0.1 * torch.randn(D, generator=gen)) for _ in range(2)) if norm else (None, None)
    rot = M.Rotation(rd, axes=axes, layout=binding.ROTATE_PAIRS if pairs else binding.ROTATE_HALVES)
    p = M.PagedParams(B, h, N, D, pages, T, width, binding.BF16 if dtype is BF16 else binding.F32,
                      kv_heads=kv, prefix_tokens=prefix, norm_eps=1e-5)

    def ints(x):
        return None if x is None else torch.as_tensor(x, dtype=torch.int32).cuda()

    start = torch.full_like(new["q"], 7.0)
    q_out = dev["q"] if in_place else strided(start, memory)
    untouched = new["q"] if in_place else start
    M.mosaic_bsa_paged_append(p, rot, ints(positions), dev["q"], dev["k"], dev["v"],
                              None if wq is None else wq.cuda(), None if wk is None else wk.cuda(),
                              ints(q_lens), ints(k_lens), table.cuda(), ints(None if prefix_len is None else [prefix_len]),
                              q_out, pool["k"], pool["v"])
    torch.cuda.synchronize()

    # the same through the entry points for contiguous tensors
    place = torch.tensor(kl).unsqueeze(1) - torch.tensor(ql).unsqueeze(1) + torch.arange(N)
    pos = torch.as_tensor(positions) if positions is not None else (P + place).unsqueeze(-1)
    pos = pos.unsqueeze(0).expand(B, -1, -1) if pos.dim() == 2 else pos
    hp = M.HeadsParams(B, N, h, D, p.dtype, kv_heads=kv, norm_eps=1e-5)
    src = {n: new[n].cuda() for n in "qk"}
    qs, ks = torch.empty_like(src["q"]), torch.empty_like(src["k"])
    at = pos.to(torch.int32).contiguous().cuda()
    if norm:
        M.mosaic_bsa_qk_norm_rope_fwd(hp, rot, at, src["q"], src["k"], wq.cuda(), wk.cuda(), qs, ks)
    else:
        M.mosaic_bsa_rope_fwd(hp, rot, at, src["q"], src["k"], qs, ks)
    want_q, want_k, want_v = untouched.clone(), pools["k"].clone(), pools["v"].clone()
    qs, ks = qs.cpu(), ks.cpu()
    for b in range(B):
        want_q[b, :, :ql[b]] = qs[b, :, :ql[b]]
        for i in range(ql[b]):
            o = int(place[b, i])
            if o < 0 or (b, o // T) in bad:
                continue
            page = int(named[b, o // T])
            want_k[page, :, o % T], want_v[page, :, o % T] = ks[b, :, i], new["v"][b, :, i]
    assert same_bits(q_out.cpu(), want_q)
    assert same_bits(pool["k"].cpu(), want_k)
    assert same_bits(pool["v"].cpu(), want_v)

    # the definition in 64 bits: norms good to (D / 2 + 8) roundings, the rotation to 8 of the pair's length
    freq = [10000.0 ** (-2.0 * i / (rd // axes)) for i in range(rd // axes // 2)] if rd else []
    for name, got, w in (("q", qs, wq), ("k", ks, wk)):
        x = new[name].double()
        z = normed(x, w, 1e-5) if norm else x
        ref = rotate(z, pos, freq, 1.0, rd, axes, pairs)
        size = z.abs().amax(-1, keepdim=True) * math.sqrt(2.0)
        tol = (8.0 + (D / 2 + 8 if norm else 0)) * U32 * size + ref.abs() * HALF_STEP[dtype] + 1e-30
        share = float(((got.double() - ref).abs() / tol).max())
        assert share <= 1.0, f"{name}: {share} of the bound"


@TYPES
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("D,rd,pairs,h,kv", [(32, 24, True, 3, 3), (64, 64, False, 8, 2), (64, 62, False, 2, 1),
                                             (128, 128, True, 16, 2), (128, 64, False, 5, 5), (64, 0, False, 4, 2)])
def test_single_tokens(dtype, norm, D, rd, pairs, h, kv):
    run(dtype, 5, h, kv, 1, D, 16, None, [1, 16, 17, 40, 64], 4, prefix=1000, rd=rd, pairs=pairs, norm=norm, seed=D)


@TYPES
@pytest.mark.parametrize("T", [1, 2, 8, 32, 128])
@pytest.mark.parametrize("norm", [False, True])
def test_chunks_of_their_own_lengths(dtype, T, norm):
    w = -(-130 // T)
    run(dtype, 6, 4, 2, 37, 64, T, [37, 0, 1, 20, 36, 5], [37, 9, 130, 128, 100, 5], w, norm=norm, seed=T)
    # tokens before the sequence's own are not written; lengths are held to what there is
    run(dtype, 5, 4, 2, 9, 64, T, [9, 9, 12, -1, 4], [3, 0, 1000, 5, -2], w, prefix=4, norm=norm, seed=T + 1)


@TYPES
@pytest.mark.parametrize("memory", ["heads", "tokens", "gaps"])
@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_memory_layouts(dtype, memory, order):
    run(dtype, 2, 6, 2, 21, 64, 8, [21, 13], [30, 14], 4, memory=memory, order=order, norm=True, seed=1)


@TYPES
def test_positions_that_are_given(dtype):
    gen = torch.Generator().manual_seed(1)
    grid = torch.randint(0, 500, (2, 19, 2), generator=gen, dtype=torch.int32)
    run(dtype, 2, 4, 2, 19, 64, 8, [19, 7], [19, 30], 4, axes=2, positions=grid, seed=2)
    run(dtype, 2, 4, 2, 19, 64, 8, [19, 7], [19, 30], 4, axes=2, positions=grid[0], pairs=True, norm=True, seed=3)
    run(dtype, 2, 4, 2, 19, 64, 8, None, [19, 30], 4, positions=grid[..., :1].contiguous() - 250, seed=4)


@TYPES
@pytest.mark.parametrize("prefix_len", [None, 0, 17, 5000, -3])
def test_places_behind_a_prefix(dtype, prefix_len):
    run(dtype, 3, 4, 2, 3, 64, 8, [3, 2, 3], [3, 30, 1], 4, prefix=900, prefix_len=prefix_len, norm=True, seed=5)


@TYPES
def test_entries_that_name_no_page(dtype):
    run(dtype, 3, 4, 2, 20, 64, 8, None, [20, 24, 32], 4, bad=((0, 0), (1, 2), (2, 1), (2, 2)), seed=6)


def test_in_place():
    run(BF16, 3, 4, 2, 20, 64, 8, [20, 3, 0], [20, 24, 32], 4, in_place=True, norm=True, seed=7)


def test_pages_past_32_bit_offsets():
    M, _ = lib()
    T, kv, D = 256, 4, 128
    pages = (1 << 32) // (T * kv * D) + 8
    k, v = (torch.zeros(pages, kv, T, D, dtype=BF16, device="cuda") for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, kn, vn = (torch.randn(2, n, 1, D, generator=gen, device="cuda").to(BF16) for n in (8, kv, kv))
    table = torch.tensor([[pages - 1, pages - 2], [3, 4]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([300, 300], dtype=torch.int32, device="cuda")
    p = M.PagedParams(2, 8, 1, D, pages, T, 2, kv_heads=kv)
    q_out = torch.empty_like(q)
    M.mosaic_bsa_paged_append(p, M.Rotation(0), None, q, kn, vn, None, None, None, lens, table, None, q_out, k, v)
    for b, page in ((0, pages - 2), (1, 4)):
        assert torch.equal(k[page, :, 43], kn[b, :, 0]) and torch.equal(v[page, :, 43], vn[b, :, 0])
        k[page, :, 43], v[page, :, 43] = 0.0, 0.0
    assert int(k.count_nonzero()) == 0 and int(v.count_nonzero()) == 0


def test_captured_steps():
    """A captured append that advances with the lengths."""
    M, _ = lib()
    B, h, kv, D, T, w = 4, 8, 2, 64, 8, 5
    gen = torch.Generator(device="cuda").manual_seed(4)
    pages = B * w
    table = torch.randperm(pages, generator=gen, device="cuda").view(B, w).to(torch.int32)
    new = [torch.randn(B, n, 1, D, generator=gen, device="cuda").to(BF16) for n in (h, kv, kv)]
    p, rot = M.PagedParams(B, h, 1, D, pages, T, w, kv_heads=kv), M.Rotation(D)
    lens = torch.tensor([1, 7, 8, 20], dtype=torch.int32, device="cuda")
    pools = [[torch.zeros(pages, kv, T, D, dtype=BF16, device="cuda") for _ in range(2)] for _ in range(2)]
    outs = [torch.empty_like(new[0]) for _ in range(2)]

    def call(i):
        M.mosaic_bsa_paged_append(p, rot, None, *new, None, None, None, lens, table, None, outs[i], *pools[i])

    call(0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(0)
    call(1)
    for _ in range(5):
        lens += 3
        for t in new:
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        g.replay()
        call(1)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and all(torch.equal(a, b) for a, b in zip(*pools))
