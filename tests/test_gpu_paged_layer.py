"""Append and attention together, as a server of ensemble members calls them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [
    dict(), dict(members=5, shared=77, own=20, heads=5, kv_heads=1, head_dim=128, window=16, sinks=1, page=8),
    dict(members=2, shared=33, own=9, heads=2, kv_heads=2, head_dim=32, window=64, sinks=0, page=16),
    dict(members=20, shared=400, own=12, heads=8, kv_heads=2, head_dim=128, window=1000, sinks=0, page=32)])
def test_members_against_whole_sequences(kw):
    from examples.local_layer import run_members
    # Both round q, k, v, the attention's weights and outputs and y to bf16, of which the weights'
    # and the products' order of sums differ: outputs of the attention within 2 steps of 2^-8, a
    # projection of them, and a last rounding
    assert run_members(**kw) <= 4 * 2.0 ** -8


def test_captured_steps_of_members():
    """A member step captured into a graph gives the eager result at every replay."""
    from examples.local_layer import LocalLayer, MemberServer
    layer = LocalLayer(128, 4, 2, 64, 1 << 20, 0)      # everything before is visible
    gen = torch.Generator().manual_seed(3)
    start = torch.randn(300, 128, generator=gen).to(torch.bfloat16).cuda()
    x = torch.randn(6, 10, 128, generator=gen).to(torch.bfloat16).cuda()
    eager, server = MemberServer(layer, 6, 300, 10), MemberServer(layer, 6, 300, 10)
    eager.begin(start)
    server.begin(start)
    want = [eager.step(x[:, t]) for t in range(10)]
    inp = x[:, 0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        server.step(inp)                               # (first call outside the capture)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = server.step(inp)
    server.length.zero_()
    for t in range(10):
        inp.copy_(x[:, t])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[t]), t


def test_a_second_beginning():
    """What members read after one beginning is forgotten at the next."""
    from examples.local_layer import LocalLayer, MemberServer
    layer = LocalLayer(128, 4, 2, 64, 1 << 20, 0)
    gen = torch.Generator().manual_seed(5)
    starts = torch.randn(2, 300, 128, generator=gen).to(torch.bfloat16).cuda()
    x = torch.randn(6, 10, 128, generator=gen).to(torch.bfloat16).cuda()
    once, twice = MemberServer(layer, 6, 300, 10), MemberServer(layer, 6, 300, 10)
    twice.begin(starts[0])
    for t in range(7):
        twice.step(x[:, t])
    for server in (once, twice):
        server.begin(starts[1])
    for t in range(10):
        assert torch.equal(twice.step(x[:, t]), once.step(x[:, t])), t
