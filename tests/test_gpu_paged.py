"""Attention over a cache in pages on the GPU against the definition in 64 bits, at the lengths,
pages, masks and layouts where tiles meet."""
import pytest
import torch

from tests.paged_reference import BF16, FP32, Cache, check, strided

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [BF16, FP32], ids=["bf16", "fp32"])


def run(dtype, B, h, kv, N, D, T, own, prefix=0, q_lens=None, left=-1, sinks=0, memory="heads",
        order="heads", bad=(), seed=0, scale=0.0, amplitude=1.0, prefix_len=None, width=None,
        k_lens=None):
    import paper_2604_16429_amd as M
    from paper_2604_16429_amd import binding
    gen = torch.Generator().manual_seed(2000 + seed)
    cache = Cache(gen, dtype, kv, T, D, own, prefix, order, bad, width)
    q = (torch.randn(B, h, N, D, generator=gen) * amplitude).to(dtype)
    q64, ql = q.double(), [N] * B if q_lens is None else q_lens
    for b in range(B):
        q[b, :, max(ql[b], 0):] = float("nan")          # what is no query may hold anything
    q = strided(q, memory)
    p = M.PagedParams(B, h, N, D, cache.pages, T, cache.width,
                      binding.BF16 if dtype is BF16 else binding.F32, kv_heads=kv, prefix_tokens=prefix,
                      window_left=left, n_sink=sinks, softmax_scale=scale)

    def ints(x):
        return None if x is None else torch.tensor(x, dtype=torch.int32).cuda()

    table, prefix_table = cache.tables()
    k_lens = list(own) if k_lens is None else k_lens
    lens = ints(q_lens), ints(k_lens)
    P = ints(None if prefix_len is None else [prefix_len])
    n = M.mosaic_bsa_paged_workspace_bytes(p)
    results = []
    for fill in (0xff, 0x00):                           # whatever the workspace holds
        ws = torch.full((max(n, 256) + 64,), fill, dtype=torch.uint8, device="cuda")
        out = torch.empty_strided(q.shape, q.stride(), dtype=dtype, device="cuda").fill_(float("nan"))
        lse = torch.full((B, h, N), float("nan"), device="cuda") if fill else None
        M.mosaic_bsa_paged_fwd(p, q, cache.k, cache.v, *lens, table, prefix_table, P, out, lse, ws,
                               workspace_bytes=n)
        torch.cuda.synchronize()
        assert bool((ws[n:] == fill).all())
        results.append((out, lse))
    assert torch.equal(results[0][0], results[1][0])    # the same bits, with and without lse
    out, lse = (x.cpu().double() for x in results[0])
    used = prefix if prefix_len is None else min(max(prefix_len, 0), prefix)
    worst = check(cache, q64, out, lse, ql, k_lens, used, dtype, left, sinks, scale)
    print(f"worst share of the bounds {worst:.3f}")


@TYPES
@pytest.mark.parametrize("D,h,kv", [(32, 2, 2), (64, 4, 2), (64, 5, 1), (128, 8, 2), (128, 16, 1), (128, 34, 2)])
def test_single_tokens(dtype, D, h, kv):
    run(dtype, 3, h, kv, 1, D, 16, [70, 1, 333], seed=D + h)


@TYPES
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300])
def test_lengths_around_the_tiles(dtype, n):
    run(dtype, 2, 4, 2, 1, 64, 8, [n, max(1, n - 1)], seed=n)
    run(dtype, 2, 4, 2, 1, 128, 32, [1, n], prefix=n, seed=n + 1)


@TYPES
@pytest.mark.parametrize("T", [1, 2, 4, 8, 16, 64, 256, 1024])
def test_pages(dtype, T):
    run(dtype, 3, 4, 2, 2, 64, T, [150, 3, 77], prefix=90, seed=T)
    run(dtype, 2, 8, 2, 20, 128, T, [150, 30], prefix=61, seed=T + 1)


@pytest.mark.parametrize("B,N,h,kv,D,P,own", [
    (24, 1, 8, 2, 64, 700, [5 * i for i in range(24)]),          # rows of all sequences fill tiles
    (3, 1, 4, 4, 128, 1025, [1, 2, 40]),
    (5, 1, 16, 2, 128, 333, [9, 0, 1, 64, 65]),                  # one has only the prefix
    (2, 1, 1, 1, 32, 257, [0, 0]),
    (40, 2, 4, 1, 64, 129, [2 + i for i in range(40)]),
    (17, 1, 8, 1, 128, 1500, [100] * 17),
    (9, 7, 5, 1, 64, 500, [7 + 13 * i for i in range(9)]),
    (4, 33, 4, 2, 128, 300, [33, 50, 100, 200]),
    (2, 150, 4, 2, 64, 200, [150, 290]),
])
@TYPES
def test_prefixes(dtype, B, N, h, kv, D, P, own):
    run(dtype, B, h, kv, N, D, 16, own, prefix=P, seed=B + P)


@pytest.mark.parametrize("dtype,B,N,h,kv,D,P,own,T", [
    # the rows of all sequences together in tiles of 16, 32 and 128, a sequence's own in 16, 32 and 128
    (BF16, 4, 1, 4, 4, 128, 4001, [1, 0, 300, 40], 16),
    (BF16, 8, 1, 16, 4, 128, 1700, [9, 700, 1, 64, 65, 0, 3, 1000], 64),
    (BF16, 17, 1, 8, 1, 128, 3003, [11 * i for i in range(17)], 8),
    (BF16, 24, 1, 8, 2, 64, 2100, [50 * i for i in range(24)], 32),
    (BF16, 40, 2, 4, 1, 64, 2500, [2 + i for i in range(40)], 256),
    (BF16, 8, 5, 8, 2, 128, 3350, [5, 7, 0, 3, 900, 64, 1, 128], 16),
    (BF16, 8, 5, 8, 2, 64, 6800, [5, 7, 0, 3, 900, 64, 1, 128], 128),
    (BF16, 8, 10, 8, 2, 128, 3377, [10, 70, 11, 33, 900, 64, 2, 128], 64),
    (BF16, 8, 12, 8, 2, 64, 6777, [12, 70, 11, 33, 900, 64, 2, 128], 8),
    (BF16, 8, 12, 8, 2, 64, 6777, [12, 70, 11, 33, 900, 64, 2, 128], 4),
    (BF16, 20, 1, 16, 8, 32, 1300, [3 * i for i in range(20)], 16),
    (FP32, 4, 1, 4, 4, 128, 2000, [1, 0, 300, 40], 16),
    (FP32, 20, 1, 8, 4, 32, 1301, [3 * i for i in range(20)], 8),
    (FP32, 9, 3, 8, 2, 64, 3001, [3 + 100 * i for i in range(9)], 64),
    (FP32, 16, 50, 16, 8, 64, 4101, [50 + i for i in range(16)], 32),
])
def test_prefixes_for_all_together(dtype, B, N, h, kv, D, P, own, T):
    """As many sequences, or as long a prefix, that it is read for all of them together."""
    q_lens = [max(0, N - b % (N + 1)) for b in range(B)]
    run(dtype, B, h, kv, N, D, T, own, prefix=P, q_lens=q_lens, order="tokens" if B == 8 else "heads", seed=B + P)
    if N < 50:
        run(dtype, B, h, kv, N, D, T, own, prefix=P, bad=[(-1, 0), (-1, (P - 1) // T), (-1, 70 // T + 1)] +
            [(b, 0) for b in (2, B - 1) if own[b]], prefix_len=P - 3, seed=B + P + 1)


@pytest.mark.parametrize("P", [0, 1, 63, 64, 1000, 2999, 3000, 9999])
def test_length_of_a_prefix_for_all_together(P):
    run(BF16, 17, 8, 1, 1, 128, 16, [11 * i for i in range(17)], prefix=3000, prefix_len=P, seed=P)


@pytest.mark.parametrize("B,most,prefix", [(65, 1500, 0), (70, 900, 300), (70, 900, 3000), (130, 1000, 0), (200, 700, 0), (1030, 40, 260)])
def test_large_batches(B, most, prefix):
    """Chunks are found by a sum over the batch."""
    own = [(37 * b * b + 11 * b) % most if b % 5 else 0 for b in range(B)]
    own[-1] = most
    run(BF16, B, 2, 1, 1, 32, 64, own, prefix=prefix, q_lens=[1 if b % 7 else 0 for b in range(B)], seed=B)


@TYPES
@pytest.mark.parametrize("N,q_lens,own,prefix", [
    (6, [6, 0, 3, 1, 5], [6, 9, 0, 1, 2], 20),           # no queries; queries that reach into the prefix
    (6, [6, 2, 0, 6, 1], [4, 0, 0, 0, 1], 0),            # more queries than tokens: some see nothing
    (5, [5, 5, 4, 1, 2], [3, 0, 1, 0, 2], 2),            # ... past the beginning of the prefix
    (130, [130, 1, 0, 64, 129], [130, 300, 5, 70, 128], 40),
    (70, [70, 3, 70, 0, 33], [10, 2, 0, 0, 200], 33),
])
def test_lengths_of_their_own(dtype, N, q_lens, own, prefix):
    run(dtype, 5, 4, 2, N, 64, 8, own, prefix=prefix, q_lens=q_lens, seed=N)
    run(dtype, 5, 4, 1, N, 128, 16, own, prefix=prefix, q_lens=q_lens, seed=N + 1)


@TYPES
def test_lengths_are_held_to_the_tables(dtype):
    run(dtype, 4, 4, 2, 2, 64, 8, [48, 48, 10, 5], prefix=40, width=6, k_lens=[100, 48, -3, 5],
        q_lens=[5, 2, -1, 1], prefix_len=-7, seed=1)
    run(dtype, 4, 4, 2, 2, 64, 8, [48, 48, 10, 5], prefix=40, width=6, k_lens=[100, 48, -3, 5],
        prefix_len=1000, seed=2)


@TYPES
@pytest.mark.parametrize("P", [0, 1, 8, 33, 64, 99, 100])
def test_prefix_length_on_the_device(dtype, P):
    run(dtype, 6, 8, 2, 1, 128, 8, [1, 5, 0, 33, 8, 100], prefix=100, prefix_len=P, seed=P)


@TYPES
@pytest.mark.parametrize("left,sinks", [(0, 0), (0, 3), (15, 0), (31, 4), (40, 50), (200, 70), (1000, 4), (64, 2**31 - 1)])
@pytest.mark.parametrize("N,prefix", [(1, 0), (1, 45), (20, 130), (100, 3)])
def test_windows(dtype, left, sinks, N, prefix):
    run(dtype, 3, 4, 2, N, 64, 8, [N, 250, N + 31], prefix=prefix, left=left, sinks=sinks, seed=left + N)
    run(dtype, 3, 4, 2, N, 128, 16, [N, 250, N + 31], prefix=prefix, left=left, sinks=sinks, seed=left + N)


@TYPES
@pytest.mark.parametrize("memory", ["heads", "tokens", "gaps"])
@pytest.mark.parametrize("order", ["heads", "tokens", "gaps"])
def test_memory_layouts(dtype, memory, order):
    run(dtype, 2, 6, 2, 3, 64, 16, [100, 20], prefix=70, memory=memory, order=order, seed=1)
    run(dtype, 2, 6, 2, 90, 128, 16, [100, 95], prefix=70, memory=memory, order=order, seed=2)


@TYPES
@pytest.mark.parametrize("N", [1, 3, 70])
def test_entries_that_name_no_page(dtype, N):
    bad = [(0, 0), (0, 5), (1, 1), (-1, 2), (-1, 0), (2, 0)]
    run(dtype, 3, 4, 1, N, 64, 8, [80, 90, 8], prefix=50, bad=bad, q_lens=[N, N, min(N, 8)], seed=N)
    run(dtype, 3, 8, 2, N, 128, 16, [80, 95, 8], prefix=50, bad=bad[1:], q_lens=[N, N, min(N, 8)], seed=N)
    # all of a sequence's pages: it sees nothing
    run(dtype, 2, 4, 2, N, 64, 16, [30, 70], bad=[(0, 0), (0, 1)], q_lens=[min(N, 30), N], seed=N)


@pytest.mark.parametrize("dtype,D", [(BF16, 32), (FP32, 32), (FP32, 64), (FP32, 128), (BF16, 64)])
@pytest.mark.parametrize("kw", [
    dict(B=8, N=70, own=[70, 71, 100, 3, 150, 64, 1, 200], q_lens=[70, 70, 69, 3, 1, 64, 0, 33], T=8),
    dict(B=8, N=70, own=[70, 71, 100, 3, 150, 64, 1, 200], q_lens=[70, 70, 69, 3, 1, 64, 0, 33], T=64, prefix=75,
         bad=[(-1, 0), (2, 1), (7, 1), (4, 0)]),
    dict(B=8, N=70, own=[70, 300, 100, 3, 150, 64, 1, 200], T=4, left=40, sinks=5),
    dict(B=16, N=50, own=[50 + 3 * b for b in range(16)], T=16, prefix=300),
    dict(B=8, N=70, own=[700, 300, 100, 3, 650, 64, 1, 200], T=32)])
def test_many_tiles_of_rows(dtype, D, kw):
    """As many as fill the chip without the tokens' being shared out."""
    run(dtype, h=32, kv=16, D=D, seed=D, **kw)


@TYPES
def test_scores_of_any_size(dtype):
    run(dtype, 2, 4, 2, 2, 64, 16, [200, 90], prefix=64, amplitude=60.0, seed=3)
    run(dtype, 2, 4, 2, 2, 128, 16, [200, 90], prefix=64, scale=1e-6, seed=4)


def test_largest_pages():
    run(BF16, 2, 4, 2, 1, 32, 65536, [300, 70], prefix=400, seed=1)
    run(FP32, 2, 4, 2, 40, 32, 65536, [300, 70], prefix=20, seed=2)
    run(BF16, 2, 4, 2, 40, 64, 65536, [300, 70], prefix=20, seed=3)


def cache_on_the_gpu(B, kv, T, D, own, prefix, dtype=BF16, spare=0):
    """A cache of torch.randn without a copy on the CPU, pages in order."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    shared, each = -(-prefix // T), -(-own // T)
    pages = shared + B * each + spare
    k, v = (torch.randn(pages, kv, T, D, generator=gen, device="cuda", dtype=dtype) for _ in range(2))
    ids = torch.arange(pages, dtype=torch.int32, device="cuda").flip(0)
    return k, v, ids[shared:shared + B * each].view(B, each).contiguous(), ids[:shared].contiguous()


def in_64_bits(k, v, table, tokens, q, scale):
    """One query [h, D] over `tokens` tokens of a row of a table."""
    kv, T = k.shape[1], k.shape[2]
    ids = table.long()
    y, z = (x[ids].transpose(0, 1).reshape(kv, -1, x.shape[-1])[:, :tokens].double() for x in (k, v))
    x = torch.matmul(q.double().view(kv, -1, q.shape[-1]), y.transpose(1, 2).contiguous()) * scale
    return torch.matmul(torch.softmax(x, -1), z).view(q.shape)


@TYPES
@pytest.mark.parametrize("B,own,prefix", [(1, 70001, 0), (3, 5, 40003), (2, 30001, 20001)])
def test_long_caches(dtype, B, own, prefix):
    """Keys split over many workgroups.  Bound: half a step of the weights and of the result, each at most
    relative to the largest value (weights sum to 1), and 2^-14 for sums of 70,000 in 32 bits."""
    import paper_2604_16429_amd as M
    from paper_2604_16429_amd import binding
    h, kv, D, T = 8, 2, 128, 64
    k, v, table, prefix_table = cache_on_the_gpu(B, kv, T, D, own, prefix, dtype)
    q = torch.randn(B, h, 1, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(dtype)
    p = M.PagedParams(B, h, 1, D, k.shape[0], T, table.shape[1],
                      binding.BF16 if dtype is BF16 else binding.F32, kv_heads=kv, prefix_tokens=prefix)
    ws = torch.empty(max(M.mosaic_bsa_paged_workspace_bytes(p), 256), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    lens = torch.full((B,), own, dtype=torch.int32, device="cuda")
    M.mosaic_bsa_paged_fwd(p, q, k, v, None, lens, table, prefix_table, None, out, workspace=ws)
    for b in range(B):
        whole = torch.cat([prefix_table[:prefix // T], table[b]])
        if prefix % T == 0:
            ref = in_64_bits(k, v, whole, prefix + own, q[b, :, 0], D ** -0.5)
        else:
            parts = []
            for t, n in ((prefix_table, prefix), (table[b], own)):
                ids = t.long()
                parts.append([x[ids].transpose(0, 1).reshape(kv, -1, D)[:, :n].double() for x in (k, v)])
            y, z = (torch.cat([a, c], 1) for a, c in zip(*parts))
            x = torch.matmul(q[b, :, 0].double().view(kv, -1, D), y.transpose(1, 2).contiguous()) * D ** -0.5
            ref = torch.matmul(torch.softmax(x, -1), z).view(h, D)
        half = 2.0 ** -8 if dtype is BF16 else 0.0
        mean = 6.0 * (own + prefix) ** -0.5                    # |out| of a mean of unit normals
        tol = half * mean * 2.0 + 2.0 ** -14 * mean + 2.0 ** -24
        assert float((out[b, :, 0].double() - ref).abs().max()) <= tol


def test_pages_past_32_bit_offsets():
    """The same tokens in pages beyond 2^32 elements of the pool: the same bits."""
    import paper_2604_16429_amd as M
    T, kv, D, B, h = 256, 4, 128, 2, 8
    pages = (1 << 32) // (T * kv * D) + 40                     # 8.6 GB each of k and v
    k, v = (torch.zeros(pages, kv, T, D, dtype=BF16, device="cuda") for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(3)
    for N, prefix in ((1, 1000), (1, 0), (100, 300)):
        q = torch.randn(B, h, N, D, generator=gen, device="cuda").to(BF16)
        for x in (k, v):
            x[:20] = torch.randn(20, kv, T, D, generator=gen, device="cuda").to(BF16)
            x[-20:] = x[:20]
        outs = []
        for first in (0, pages - 20):
            table = (first + torch.arange(10, dtype=torch.int32, device="cuda")).view(2, 5)
            prefix_table = first + 10 + torch.arange(-(-prefix // T), dtype=torch.int32, device="cuda")
            p = M.PagedParams(B, h, N, D, pages, T, 5, kv_heads=kv, prefix_tokens=prefix)
            lens = torch.tensor([1200, 777], dtype=torch.int32, device="cuda")
            ws = torch.empty(max(M.mosaic_bsa_paged_workspace_bytes(p), 256), dtype=torch.uint8, device="cuda")
            out = torch.empty_like(q)
            M.mosaic_bsa_paged_fwd(p, q, k, v, None, lens, table, prefix_table, None, out, workspace=ws)
            outs.append(out)
        assert torch.equal(*outs) and bool(outs[0].isfinite().all())


def test_another_stream_and_graphs_that_share_a_workspace():
    """Two captured calls with one workspace, replayed in turn with other lengths in place."""
    import paper_2604_16429_amd as M
    h, kv, D, T, B, prefix = 8, 2, 128, 16, 6, 5000
    k, v, table, prefix_table = cache_on_the_gpu(B, kv, T, D, 900, prefix)
    gen = torch.Generator(device="cuda").manual_seed(5)
    p = [M.PagedParams(B, h, n, D, k.shape[0], T, table.shape[1], kv_heads=kv, prefix_tokens=prefix)
         for n in (1, 40)]
    n = max(M.mosaic_bsa_paged_workspace_bytes(x) for x in p)
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    q = [torch.randn(B, h, x.q_tokens, D, generator=gen, device="cuda").to(BF16) for x in p]
    out = [torch.empty_like(x) for x in q]
    lens = torch.full((B,), 100, dtype=torch.int32, device="cuda")
    plen = torch.tensor([prefix], dtype=torch.int32, device="cuda")

    def call(i, to, space):
        M.mosaic_bsa_paged_fwd(p[i], q[i], k, v, None, lens, table, prefix_table, plen, to, workspace=space)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(0, out[0], ws)
        call(1, out[1], ws)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i, out[i], ws)
        graphs.append(g)
    other = torch.empty_like(ws)
    for turn in range(4):
        lens.copy_(torch.randint(40, 900, (B,), generator=gen, device="cuda", dtype=torch.int32))
        plen.fill_((5000, 7, 0, 4999)[turn])
        for i in (0, 1) if turn % 2 else (1, 0):
            out[i].fill_(float("nan"))
            graphs[i].replay()
        for i in range(2):
            want = torch.empty_like(out[i])
            call(i, want, other)
            torch.cuda.synchronize()
            assert torch.equal(out[i], want)


def test_token_strides_past_32_bits_of_a_tile():
    """Rows 2^24 elements apart: the kernels for any stride take over, with the same workspace."""
    import paper_2604_16429_amd as M
    T, kv, D, B, h = 8, 1, 64, 2, 4
    gen = torch.Generator(device="cuda").manual_seed(11)
    far = [torch.zeros(T << 24, dtype=BF16, device="cuda").as_strided((40, kv, T, D), (D, 0, 1 << 24, 1))
           for _ in range(2)]
    near = [torch.randn(40, kv, T, D, generator=gen, device="cuda").to(BF16) for _ in range(2)]
    for a, b in zip(far, near):
        a.copy_(b)
    table = torch.randperm(40, generator=gen, device="cuda")[:36].to(torch.int32)
    for N, prefix in ((50, 0), (50, 60), (1, 60)):
        q = torch.randn(B, h, N, D, generator=gen, device="cuda").to(BF16)
        p = M.PagedParams(B, h, N, D, 40, T, 14, kv_heads=kv, prefix_tokens=prefix)
        lens = torch.tensor([112, 51], dtype=torch.int32, device="cuda")
        n = M.mosaic_bsa_paged_workspace_bytes(p)
        outs = []
        for k, v in (far, near):
            ws, out = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda"), torch.empty_like(q)
            M.mosaic_bsa_paged_fwd(p, q, k, v, None, lens, table[:28].contiguous().view(2, 14), table[28:].contiguous(),
                                   None, out, workspace=ws)
            outs.append(out.float())
        # each within its roundings of the definition: weights and result, a half step each
        assert float((outs[0] - outs[1]).abs().max()) <= 2 * 2 * 2.0 ** -8 * float(near[1].abs().max())


def test_streams_as_objects():
    import paper_2604_16429_amd as M
    k, v, table, prefix_table = cache_on_the_gpu(2, 2, 16, 64, 100, 40)
    q = torch.randn(2, 4, 1, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(BF16)
    p = M.PagedParams(2, 4, 1, 64, k.shape[0], 16, table.shape[1], kv_heads=2, prefix_tokens=40)
    lens = torch.full((2,), 100, dtype=torch.int32, device="cuda")
    outs = [torch.empty_like(q) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for out, stream in zip(outs, (None, side)):
        M.mosaic_bsa_paged_fwd(p, q, k, v, None, lens, table, prefix_table, None, out, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(*outs)


@TYPES
@pytest.mark.parametrize("N", [1, 40])
def test_inputs_that_share_memory(dtype, N):
    """Key/value heads that are one (stride 0), queries that all sequences share, kv_heads left at 0."""
    import paper_2604_16429_amd as M
    from paper_2604_16429_amd import binding
    k, v, table, prefix_table = cache_on_the_gpu(3, 1, 16, 64, 100, 40, dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(1, 4, N, 64, device="cuda", generator=gen).to(dtype)
    p = M.PagedParams(3, 4, N, 64, k.shape[0], 16, table.shape[1], binding.BF16 if dtype is BF16 else binding.F32,
                      prefix_tokens=40)
    lens = torch.tensor([100, 60, 41], dtype=torch.int32, device="cuda")
    ws = torch.empty(max(M.mosaic_bsa_paged_workspace_bytes(p), 256), dtype=torch.uint8, device="cuda")
    outs = []
    for real in (False, True):
        a = [x.expand(-1, 4, -1, -1) for x in (k, v)] + [q.expand(3, -1, -1, -1)]
        a = [x.contiguous() for x in a] if real else a
        out = torch.empty(3, 4, N, 64, dtype=dtype, device="cuda")
        M.mosaic_bsa_paged_fwd(p, a[2], a[0], a[1], None, lens, table, prefix_table, None, out, workspace=ws)
        outs.append(out)
    assert torch.equal(*outs) and bool(outs[0].isfinite().all())


@pytest.mark.parametrize("dtype,B,D,P", [(FP32, 16, 128, 3001), (FP32, 64, 32, 4101), (BF16, 64, 32, 4901)])
def test_prefixes_for_all_together_beside_tiles_of_rows(dtype, B, D, P):
    """Own tokens in tiles of 128 rows through registers, the prefix's in tiles of 32."""
    run(dtype, B, 16, 8, 50, D, 32, [50 + b for b in range(B)], prefix=P, q_lens=[50 - b % 51 for b in range(B)], seed=B + D)


@pytest.mark.parametrize("dtype,B,N,P", [(BF16, 128, 15, 614), (BF16, 64, 12, 256), (FP32, 40, 12, 300)])
def test_short_prefixes_of_many_rows(dtype, B, N, P):
    """Too short to be worked on for all together beside that many rows, though that would save reads."""
    import paper_2604_16429_amd as M
    from paper_2604_16429_amd import binding
    p = M.PagedParams(B, 32, N, 128, 1000, 64, 1, binding.BF16 if dtype is BF16 else binding.F32, kv_heads=4, prefix_tokens=P)
    assert M.mosaic_bsa_paged_workspace_bytes(p) == 0
    run(dtype, B, 32, 4, N, 128, 64, [N + b % 40 for b in range(B)], prefix=P, q_lens=[N - b % (N + 1) for b in range(B)],
        seed=B + P)


@pytest.mark.parametrize("N,own,prefix", [(50, 900, 0), (10, 300, 14000), (10, 900, 14000)])
def test_token_strides_past_32_bits_with_a_workspace(N, own, prefix):
    """Rows 2^24 elements apart, where tokens are split, the prefix is worked on for all together, or both: the
    kernels for any stride leave other sums in the workspace, whose size is asked for without strides."""
    import paper_2604_16429_amd as M
    T, kv, D, B, h = 8, 1, 64, 8, 4
    each, shared = -(-own // T), prefix // T
    pages = shared + B * each
    gen = torch.Generator(device="cuda").manual_seed(12)
    near = [torch.randn(pages, kv, T, D, generator=gen, device="cuda").to(BF16) for _ in range(2)]
    far = [torch.zeros(T << 24, dtype=BF16, device="cuda").as_strided((pages, kv, T, D), (D, 0, 1 << 24, 1))
           for _ in range(2)]
    for a, b in zip(far, near):
        a.copy_(b)
    ids = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    q = torch.randn(B, h, N, D, generator=gen, device="cuda").to(BF16)
    p = M.PagedParams(B, h, N, D, pages, T, each, kv_heads=kv, prefix_tokens=prefix)
    lens = torch.tensor([own - 31 * b for b in range(B)], dtype=torch.int32, device="cuda")
    n = M.mosaic_bsa_paged_workspace_bytes(p)
    assert n > 0
    outs = []
    for k, v in (far, near):
        ws = torch.full((n + 4096,), 0xff, dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        M.mosaic_bsa_paged_fwd(p, q, k, v, None, lens, ids[shared:].contiguous().view(B, each), ids[:shared].contiguous(),
                               None, out, workspace=ws, workspace_bytes=n)
        assert bool((ws[n:] == 0xff).all())
        outs.append(out.float())
    # each within its roundings of the definition: weights and result, a half step each
    assert float((outs[0] - outs[1]).abs().max()) <= 2 * 2 * 2.0 ** -8 * float(near[1].abs().max())


@pytest.mark.parametrize("named", [True, False], ids=["given", "current"])
def test_calls_wait_for_their_stream(named):
    """Inputs that work queued on the same stream has yet to make."""
    import paper_2604_16429_amd as M
    B, h, kv, D, T, prefix, own = 3, 4, 2, 64, 16, 40, 100
    k0, v0, table, prefix_table = cache_on_the_gpu(B, kv, T, D, own, prefix)
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = [torch.randn(B, n, 1, D, device="cuda", generator=gen).to(BF16) for n in (h, kv, kv)]
    p, rot = M.PagedParams(B, h, 1, D, k0.shape[0], T, table.shape[1], kv_heads=kv, prefix_tokens=prefix), M.Rotation(D)
    lens = torch.full((B,), own, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(M.mosaic_bsa_paged_workspace_bytes(p), 256), dtype=torch.uint8, device="cuda")
    busy = torch.randn(8192, 8192, device="cuda").to(BF16)

    def serve(late, stream):
        k, v = k0.clone(), v0.clone()
        inputs = [torch.zeros_like(x) for x in new]
        turned, out = torch.zeros_like(new[0]), torch.zeros_like(new[0])
        torch.cuda.synchronize()
        with torch.cuda.stream(late):
            for _ in range(20):
                torch.mm(busy, busy)
            for x, y in zip(inputs, new):
                x.copy_(y)

        def calls():
            M.mosaic_bsa_paged_append(p, rot, None, *inputs, None, None, None, lens, table, None, turned, k, v, stream=stream)
            M.mosaic_bsa_paged_fwd(p, turned, k, v, None, lens, table, prefix_table, None, out, workspace=ws, stream=stream)

        if stream is None:
            with torch.cuda.stream(late):
                calls()
        else:
            calls()
        torch.cuda.synchronize()
        return turned, k, v, out

    want = serve(torch.cuda.current_stream(), None)
    side = torch.cuda.Stream()
    got = serve(side, side if named else None)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and bool(want[3].count_nonzero() > 0)
