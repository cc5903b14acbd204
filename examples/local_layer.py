"""A local attention layer out of the package's entry points, trained and then served.

    python -m examples.local_layer            # needs a GPU

One projection gives q, k and v of every token side by side; their heads are normed and
rotated by position in one pass, attention runs inside a sliding window with a few first
tokens that stay visible, and a second projection closes the layer.  Gradients go back the
same way, into one tensor beside the projection's output.  Then the layer reads the same
tokens one at a time: a single call norms, rotates and writes keys and values into a ring
cache that holds the window and the first tokens, and the attention reads it.  Members of an
ensemble that go on from one beginning read it once, into pages that all of them share, and keep
pages of their own for what follows.
"""
from __future__ import annotations

import argparse

import torch

import paper_2604_16429_amd as bsa
from paper_2604_16429_amd import binding


class LocalLayer:
    def __init__(self, width, heads, kv_heads, head_dim, window, sinks, seed=0):
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.window, self.sinks = window, sinks
        gen = torch.Generator().manual_seed(seed)
        all_heads = heads + 2 * kv_heads

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=gen) / cols ** 0.5).to(torch.bfloat16).cuda()

        self.w_in = weight(all_heads * head_dim, width)
        self.w_out = weight(width, heads * head_dim)
        self.q_norm = torch.ones(head_dim, device="cuda")
        self.k_norm = torch.ones(head_dim, device="cuda")
        self.rotation = bsa.Rotation(head_dim)

    def _split(self, qkv):
        """Views [B, heads, N, D] of q, k, v in a projection's output [B, N, all heads * D]."""
        x = qkv.view(*qkv.shape[:2], -1, self.head_dim).transpose(1, 2)
        return x.split([self.heads, self.kv_heads, self.kv_heads], dim=1)

    def _params(self, batch, tokens):
        heads = bsa.HeadsParams(batch, tokens, self.heads, self.head_dim, binding.BF16,
                                kv_heads=self.kv_heads)
        window = bsa.WindowParams(batch, self.heads, tokens, tokens, self.head_dim, binding.BF16,
                                  kv_heads=self.kv_heads, window_left=self.window - 1,
                                  n_sink=self.sinks)
        return heads, window

    def forward(self, x):
        """x [B, N, width] -> (y [B, N, width], what the backward needs)."""
        B, N, _ = x.shape
        hp, wp = self._params(B, N)
        qkv = (x.flatten(0, 1) @ self.w_in.t()).view(B, N, -1)
        q, k, v = self._split(qkv)
        qr = torch.empty(B, self.heads, N, self.head_dim, dtype=x.dtype, device="cuda")
        kr = torch.empty(B, self.kv_heads, N, self.head_dim, dtype=x.dtype, device="cuda")
        bsa.mosaic_bsa_qk_norm_rope_fwd(hp, self.rotation, None, q, k, self.q_norm, self.k_norm, qr,
                                        kr)
        out = torch.empty(B, N, self.heads, self.head_dim, dtype=x.dtype, device="cuda")
        lse = torch.empty(B, self.heads, N, device="cuda")
        ws = _space(bsa.mosaic_bsa_window_workspace_bytes(wp, binding.OP_FWD))
        bsa.mosaic_bsa_window_fwd(wp, qr, kr, v, out.transpose(1, 2), lse, workspace=ws)
        y = (out.view(B * N, -1) @ self.w_out.t()).view(B, N, -1)
        return y, (x, qkv, qr, kr, out, lse)

    def backward(self, dy, saved):
        """Gradients of x, w_in, w_out and the two norms' weights."""
        x, qkv, qr, kr, out, lse = saved
        B, N, _ = x.shape
        hp, wp = self._params(B, N)
        dy2 = dy.reshape(B * N, -1)
        dout = (dy2 @ self.w_out).view(B, N, self.heads, self.head_dim).transpose(1, 2)
        q, k, v = self._split(qkv)
        dqkv = torch.empty_like(qkv)
        dq, dk, dv = self._split(dqkv)
        dqr, dkr = torch.empty_like(qr), torch.empty_like(kr)
        ws = _space(bsa.mosaic_bsa_window_workspace_bytes(wp, binding.OP_BWD))
        bsa.mosaic_bsa_window_bwd(wp, qr, kr, v, out.transpose(1, 2), lse, dout, dqr, dkr, dv, ws)
        dqn, dkn = torch.empty_like(self.q_norm), torch.empty_like(self.k_norm)
        ws = _space(bsa.mosaic_bsa_qk_norm_rope_workspace_bytes(hp))
        bsa.mosaic_bsa_qk_norm_rope_bwd(hp, self.rotation, None, q, k, self.q_norm, self.k_norm, dqr,
                                        dkr, dq, dk, dqn, dkn, ws)
        dqkv2 = dqkv.view(B * N, -1)
        return ((dqkv2 @ self.w_in).view_as(x), dqkv2.t() @ x.flatten(0, 1),
                dy2.t() @ out.view(B * N, -1), dqn, dkn)


class Server:
    """Reads tokens one at a time; the cache holds the window and the first tokens."""

    def __init__(self, layer, batch):
        self.layer, self.batch = layer, batch
        rows, ring = layer.sinks + layer.window, layer.window
        self.k_cache, self.v_cache = (
            torch.zeros(batch, layer.kv_heads, rows, layer.head_dim, dtype=torch.bfloat16,
                        device="cuda") for _ in range(2))
        self.length = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.hp = bsa.HeadsParams(batch, 1, layer.heads, layer.head_dim, binding.BF16,
                                  kv_heads=layer.kv_heads, cache_tokens=rows)
        self.wp = bsa.WindowParams(batch, layer.heads, 1, rows, layer.head_dim, binding.BF16,
                                   kv_heads=layer.kv_heads, window_left=layer.window - 1,
                                   n_sink=layer.sinks, ring=ring)
        self.ws = _space(bsa.mosaic_bsa_window_workspace_bytes(self.wp, binding.OP_FWD))
        self.q = torch.empty(batch, layer.heads, 1, layer.head_dim, dtype=torch.bfloat16,
                             device="cuda")
        self.out = torch.empty_like(self.q)

    def step(self, x):
        """x [B, width] -> y [B, width]."""
        lay = self.layer
        q, k, v = lay._split((x @ lay.w_in.t()).view(self.batch, 1, -1))
        late = lay.sinks + (self.length - lay.sinks) % lay.window
        rows = torch.where(self.length < lay.sinks, self.length, late).to(torch.int32)
        bsa.mosaic_bsa_qk_norm_rope_fwd(self.hp, lay.rotation, self.length.view(-1, 1), q, k,
                                        lay.q_norm, lay.k_norm, self.q, self.k_cache, v=v,
                                        v_out=self.v_cache, rows=rows)
        self.length += 1
        bsa.mosaic_bsa_window_fwd(self.wp, self.q, self.k_cache, self.v_cache, self.out,
                                  k_lens=self.length, workspace=self.ws)
        return self.out.view(self.batch, -1) @ lay.w_out.t()


class MemberServer:
    """Members that go on from one common beginning, which is read and kept once: pages of a pool, those
    of the beginning in `prefix_table`, each member's own, for `own` tokens, in its row of `table`."""

    def __init__(self, layer, members, shared, own, page=64):
        self.layer, self.members, self.shared, self.page = layer, members, shared, page
        n, each = -(-shared // page), -(-own // page)
        self.pages = n + members * each
        ids = torch.arange(self.pages, dtype=torch.int32, device="cuda")
        self.prefix_table, self.table = ids[:n].contiguous(), ids[n:].view(members, each).contiguous()
        self.k_pages, self.v_pages = (
            torch.zeros(self.pages, layer.kv_heads, page, layer.head_dim, dtype=torch.bfloat16,
                        device="cuda") for _ in range(2))
        self.length = torch.zeros(members, dtype=torch.int32, device="cuda")
        self.steps = self._params(members, 1, each, shared)
        self.ws = _space(bsa.mosaic_bsa_paged_workspace_bytes(self.steps))

    def _params(self, batch, tokens, table_pages, prefix):
        lay = self.layer
        return bsa.PagedParams(batch, lay.heads, tokens, lay.head_dim, self.pages, self.page,
                               table_pages, binding.BF16, kv_heads=lay.kv_heads, prefix_tokens=prefix,
                               window_left=lay.window - 1, n_sink=lay.sinks)

    def _run(self, p, x, lengths, table, prefix_table, ws):
        """x [batch, tokens, width], counted in `lengths` already."""
        lay, (B, N, _) = self.layer, x.shape
        q, k, v = lay._split((x.reshape(B * N, -1) @ lay.w_in.t()).view(B, N, -1))
        qr = torch.empty(B, lay.heads, N, lay.head_dim, dtype=x.dtype, device="cuda")
        bsa.mosaic_bsa_paged_append(p, lay.rotation, None, q, k, v, lay.q_norm, lay.k_norm, None,
                                    lengths, table, None, qr, self.k_pages, self.v_pages)
        out = torch.empty(B, N, lay.heads, lay.head_dim, dtype=x.dtype, device="cuda")
        bsa.mosaic_bsa_paged_fwd(p, qr, self.k_pages, self.v_pages, None, lengths, table,
                                 prefix_table, None, out.transpose(1, 2), workspace=ws)
        return (out.view(B * N, -1) @ lay.w_out.t()).view(B, N, -1)

    def begin(self, x):
        """x [shared, width], the common beginning -> y [shared, width].  Members have nothing of their own yet."""
        self.length.zero_()
        p = self._params(1, self.shared, self.prefix_table.numel(), 0)
        lengths = torch.full((1,), self.shared, dtype=torch.int32, device="cuda")
        ws = _space(bsa.mosaic_bsa_paged_workspace_bytes(p))
        return self._run(p, x.unsqueeze(0), lengths, self.prefix_table.view(1, -1), None, ws)[0]

    def step(self, x):
        """x [members, width] -> y [members, width]; up to `own` times (a captured step counts on the GPU, so
        that the host cannot refuse one more, which would take the place of the last)."""
        self.length += 1
        return self._run(self.steps, x.unsqueeze(1), self.length, self.table, self.prefix_table, self.ws)[:, 0]


def _space(n):
    return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")


def run(batch=2, tokens=600, width=256, heads=8, kv_heads=2, head_dim=64, window=128, sinks=4,
        steps=6, rate=0.02):
    """Trains the layer to repeat its input and reads the tokens again one by one.  Returns the
    losses and the largest difference of the two ways, relative to the largest output."""
    layer = LocalLayer(width, heads, kv_heads, head_dim, window, sinks)
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(batch, tokens, width, generator=gen).to(torch.bfloat16).cuda()
    losses = []
    for _ in range(steps):
        y, saved = layer.forward(x)
        diff = y.float() - x.float()
        losses.append(float(diff.square().mean()))
        dy = (diff * (2.0 / diff[..., 0].numel())).to(torch.bfloat16)
        _, dw_in, dw_out, dqn, dkn = layer.backward(dy, saved)
        for w, g in ((layer.w_in, dw_in), (layer.w_out, dw_out), (layer.q_norm, dqn),
                     (layer.k_norm, dkn)):
            # a step of `rate` of the weights' length down the gradient
            w -= (rate * w.float().norm() / g.float().norm()) * g
    whole, _ = layer.forward(x)
    server = Server(layer, batch)
    one_by_one = torch.stack([server.step(x[:, t]) for t in range(tokens)], dim=1)
    apart = float((whole.float() - one_by_one.float()).abs().max() / whole.float().abs().max())
    return losses, apart


def run_members(members=3, shared=300, own=40, width=256, heads=8, kv_heads=2, head_dim=64, window=128,
                sinks=4, page=64):
    """Members that go on from a common beginning, token by token from pages, against whole sequences:
    the largest difference relative to the largest output."""
    layer = LocalLayer(width, heads, kv_heads, head_dim, window, sinks)
    gen = torch.Generator().manual_seed(2)
    start = torch.randn(shared, width, generator=gen).to(torch.bfloat16).cuda()
    rest = torch.randn(members, own, width, generator=gen).to(torch.bfloat16).cuda()
    whole, _ = layer.forward(torch.cat([start.expand(members, -1, -1), rest], dim=1))
    server = MemberServer(layer, members, shared, own, page)
    y = server.begin(start)
    steps = torch.stack([server.step(rest[:, t]) for t in range(own)], dim=1)
    apart = torch.cat([(whole[0, :shared].float() - y.float()).abs().flatten(),
                       (whole[:, shared:].float() - steps.float()).abs().flatten()])
    return float(apart.max() / whole.float().abs().max())


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("batch", 2), ("tokens", 600), ("width", 256), ("heads", 8), ("kv-heads", 2),
                        ("head-dim", 64), ("window", 128), ("sinks", 4), ("steps", 6)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    losses, apart = run(a.batch, a.tokens, a.width, a.heads, a.kv_heads, a.head_dim, a.window, a.sinks,
                        a.steps)
    print("loss by step:", " ".join(f"{x:.4f}" for x in losses))
    print(f"whole sequence against single tokens: {apart:.2e} of the largest output")
    apart = run_members(3, a.tokens, 40, a.width, a.heads, a.kv_heads, a.head_dim, a.window, a.sinks)
    print(f"members on a common beginning, from pages: {apart:.2e} of the largest output")
