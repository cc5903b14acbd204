"""The example layer: training lowers its loss, and reading token by token through the ring
cache gives what the whole sequence gives."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(), dict(tokens=90, heads=5, kv_heads=1, head_dim=128, window=16, sinks=1),
                                dict(batch=1, tokens=40, heads=2, kv_heads=2, head_dim=32, window=64, sinks=0)])
def test_layer(kw):
    from examples.local_layer import run
    losses, apart = run(**kw)
    assert losses[-1] < losses[0]
    # Both round q, k, v, the attention's weights and outputs and y to bf16, of which the weights'
    # and the products' order of sums differ: outputs of the attention within 2 steps of 2^-8, a
    # projection of them, and a last rounding
    assert apart <= 4 * 2.0 ** -8


def test_captured_steps_replay():
    """A decoding step captured into a graph gives the eager result at every replay, with eager
    work between the replays."""
    from examples.local_layer import LocalLayer, Server
    layer = LocalLayer(128, 4, 2, 64, 64, 2)
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(2, 20, 128, generator=gen).to(torch.bfloat16).cuda()
    eager, server = Server(layer, 2), Server(layer, 2)
    want = [eager.step(x[:, t]) for t in range(20)]
    inp = x[:, 0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            server.step(inp)                           # (first calls outside the capture)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = server.step(inp)
    server.length.zero_()
    for t in range(20):
        inp.copy_(x[:, t])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[t]), t


def test_captured_training_pass_replays():
    import paper_2604_16429_amd as M
    from paper_2604_16429_amd import binding
    gen = torch.Generator().manual_seed(4)
    B, h, kv, n, D = 2, 4, 2, 300, 64
    p = M.WindowParams(B, h, n, n, D, binding.BF16, kv_heads=kv, window_left=63, n_sink=4)

    def rand(heads):
        return torch.randn(B, heads, n, D, generator=gen).to(torch.bfloat16).cuda()

    q, k, v, do = rand(h), rand(kv), rand(kv), rand(h)
    ws = torch.empty(max(256, M.mosaic_bsa_window_workspace_bytes(p, binding.OP_FWD)), dtype=torch.uint8,
                     device="cuda")
    wb = torch.empty(M.mosaic_bsa_window_workspace_bytes(p, binding.OP_BWD), dtype=torch.uint8, device="cuda")

    def outputs():
        return (torch.empty_like(q), torch.empty(B, h, n, device="cuda"), torch.empty_like(q),
                torch.empty_like(k), torch.empty_like(v))

    def run(o):
        M.mosaic_bsa_window_fwd(p, q, k, v, o[0], o[1], workspace=ws)
        M.mosaic_bsa_window_bwd(p, q, k, v, o[0], o[1], do, o[2], o[3], o[4], wb)

    eager, held = outputs(), outputs()
    run(held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(held)
    for i in range(4):
        for t, heads in ((q, h), (k, kv), (v, kv), (do, h)):
            t.copy_(rand(heads))
        run(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, held):
            assert torch.equal(a, b), i
