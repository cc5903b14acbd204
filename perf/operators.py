"""Position rotation, head norms and windowed attention, as cases that can be timed.

Three operators that sit next to the block-sparse attention of this package:

  rope     the position rotation of queries and keys (mosaic_bsa_rope_*), one or two
           coordinates a token, halves or neighbouring pairs, a part of the head,
           frequencies stretched for long contexts;
  norm     the root-mean-square norm of each query and key head with the rotation in
           the same pass (mosaic_bsa_qk_norm_rope_*), for single tokens straight into
           the cache;
  window   attention inside a sliding window with a few first tokens that stay visible
           (mosaic_bsa_window_*): whole sequences, chunks and single tokens over a cache.

A case's "op" is the operator with its direction: "_fwd", "_bwd" or "_train" (forward,
then backward).  `run` computes either the plain form (elementary torch operations in
32 bits, angles in 64) or, where `own` is true, calls the package.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------ the cases

def _heads(op, dtype, batch, tokens, heads, kv_heads, head_dim, rotary_dim, layout, axes=1,
           scaling="none", factor=1.0, original=0, far=0, memory="packed", cache=0, name=None):
    """A rope or norm case.  layout: "halves" (channel c with c + half) or "pairs" (2c with
    2c + 1).  far: positions start at a token below this one (0: at 0).  memory: "packed"
    (q, k, v side by side for each token, as one projection leaves them) or "heads"
    ([B, h, N, D]).  cache: rows of a key/value cache that the new keys and values go to."""
    c = dict(op=op, dtype=dtype, batch=batch, tokens=tokens, heads=heads, kv_heads=kv_heads,
             head_dim=head_dim, rotary_dim=rotary_dim, layout=layout, axes=axes, scaling=scaling,
             factor=factor, original=original, far=far, memory=memory, cache=cache)
    if name:
        c["name"] = name
    return c


def _window(op, dtype, batch, heads, kv_heads, q_tokens, k_tokens, head_dim, left, right, sinks,
            ring=0, ragged=False, memory="packed", name=None):
    """A window case: query p sees key j where j <= p + right and (j >= p - left or
    j < sinks).  The last query stands at the last key.  left, right -1: no bound.  ring:
    rows of the cache behind the sinks, reused in turn.  ragged: every sequence of the
    batch has a length of its own.  memory: "packed", "heads" or "tokens" ([B, N, h, D])."""
    c = dict(op=op, dtype=dtype, batch=batch, heads=heads, kv_heads=kv_heads, q_tokens=q_tokens,
             k_tokens=k_tokens, head_dim=head_dim, left=left, right=right, sinks=sinks, ring=ring,
             ragged=ragged, memory=memory)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One new token of one sequence: two small heads tensors, latency only.
        _heads("rope_fwd", "bf16", 1, 1, 20, 5, 64, 64, "pairs", far=28800, memory="heads",
               name="rope_step"),
        # Queries and keys of the 1.5 degree grid by latitude and longitude index, as the
        # projection of a layer leaves them.
        _heads("rope_fwd", "bf16", 4, 28800, 16, 16, 64, 64, "halves", axes=2,
               name="rope_grid15"),
        # Gradients of a long sequence in full precision, half of each head rotated, with
        # frequencies stretched to eight times the trained length.
        _heads("rope_bwd", "fp32", 1, 131072, 16, 4, 64, 32, "halves", scaling="ramp", factor=8.0,
               original=16384, memory="heads", name="rope_long_bwd"),
        # One token of each of 24 members: norms, rotation, and keys and values into a cache.
        _heads("norm_fwd", "bf16", 24, 1, 16, 4, 128, 128, "halves", far=4000, cache=4100,
               name="norm_step"),
        # Training pass over the 1.5 degree grid at head dim 128, grouped heads.
        _heads("norm_train", "bf16", 4, 28800, 16, 4, 128, 128, "halves", name="norm_grid15_train"),
        # A small study in full precision: odd length, neighbouring pairs, most of the head.
        _heads("norm_train", "fp32", 3, 1001, 6, 2, 32, 24, "pairs", scaling="base", factor=4.0,
               far=100000, memory="heads", name="norm_odd_fp32_train"),
        # One new token of one sequence over the last 1,024 and 4 first ones.
        _window("window_fwd", "bf16", 1, 8, 8, 1, 2048, 64, 1023, 0, 4, memory="tokens",
                name="window_step"),
        # One new token of each of 24 members over ring caches of different lengths.
        _window("window_fwd", "bf16", 24, 16, 4, 1, 4100, 128, 4095, 0, 4, ring=4096, ragged=True,
                memory="heads", name="window_step_ring"),
        # A chunk of up to 100 new tokens on long caches (head dim 64, 5 query heads per key head).
        _window("window_fwd", "bf16", 4, 20, 4, 100, 28800, 64, 1999, 0, 5, ragged=True,
                memory="heads", name="window_chunk"),
        # A whole long sequence: 131,072 tokens, window of 4,096.
        _window("window_fwd", "bf16", 1, 16, 4, 131072, 131072, 128, 4095, 0, 4,
                name="window_long"),
        # Training pass on the 1.5 degree grid in token order, window of 1,024.
        _window("window_train", "bf16", 4, 16, 4, 28800, 28800, 128, 1023, 0, 4,
                name="window_grid15_train"),
        # A small study in full precision: both sides visible, lengths of their own.
        _window("window_train", "fp32", 2, 8, 2, 1501, 1501, 32, 200, 200, 1, ragged=True,
                memory="tokens", name="window_ragged_fp32_train"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn_heads(rng):
    op = rng.choice(["rope_fwd", "rope_bwd", "norm_fwd", "norm_train"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    kv = rng.randint(1, 8)
    heads = kv * rng.choice([1, 1, 2, 4, 5])
    D = rng.choice([32, 64, 64, 128])
    axes = rng.choice([1, 1, 2])
    rd = rng.choice([D, D, D // 2, D - 8])
    scaling = rng.choice(["none", "none", "linear", "base", "ramp"]) if axes == 1 else "none"
    if rng.random() < 0.3:                        # a decoding step
        batch, tokens, cache = _log_int(rng, 1, 64), 1, 0
        if op == "norm_fwd":
            cache = _log_int(rng, 64, 4100)
    else:
        batch, tokens, cache = _log_int(rng, 1, 24), _log_int(rng, 2, 131072), 0
    return _heads(op, dtype, batch, tokens, heads, kv, D, rd, rng.choice(["halves", "pairs"]),
                  axes, scaling, 1.0 if scaling == "none" else float(rng.choice([2, 4, 8])),
                  16384 if scaling == "ramp" else 0,
                  0 if axes == 2 else rng.choice([0, 4000, 100000]),
                  rng.choice(["packed", "heads"]), cache)


def _drawn_window(rng):
    op = rng.choice(["step", "step", "chunk", "whole", "train", "train"])
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    kv = rng.randint(1, 8)
    heads = kv * rng.choice([1, 1, 2, 4, 5])
    D = rng.choice([32, 64, 64, 128])
    left = _log_int(rng, 16, 4096) - 1
    sinks = rng.choice([0, 1, 4, 4, 5, 64])
    ragged = rng.random() < 0.5
    if op in ("step", "chunk"):
        nq = 1 if op == "step" else rng.randint(2, 128)
        ring = 0
        nk = max(_log_int(rng, 64, 65536), nq)
        if rng.random() < 0.4:
            ring = left + nq + rng.choice([0, 1, 100])
            nk = sinks + ring
            ragged = True                         # lengths past the ring
        return _window("window_fwd", dtype, _log_int(rng, 1, 32), heads, kv, nq, nk, D, left, 0,
                       sinks, ring, ragged, rng.choice(["heads", "tokens"]))
    n = _log_int(rng, 33, 131072 if op == "whole" else 28800)
    return _window("window_fwd" if op == "whole" else "window_train", dtype, _log_int(rng, 1, 4),
                   heads, kv, n, n, D, left, rng.choice([0, 0, 0, left]), sinks, 0, ragged,
                   rng.choice(["packed", "heads", "tokens"]))


def draw(rng):
    """One more case: any operator, direction, type, layout and length that the listed ones
    stand for, at most as much work as the largest of them (an eighth of it in fp32)."""
    while True:
        c = _drawn_heads(rng) if rng.random() < 0.4 else _drawn_window(rng)
        w = work(c)
        share = 8.0 if c["dtype"] == "fp32" else 1.0
        if w["bytes"] <= 3.0e9 and w["flops"] <= 4.0e12 / share:
            return c


# ------------------------------------------------------------------ inputs

def _lengths(c, seed):
    """(query lengths, key lengths) of the batch as lists.  The lengths of a ragged batch
    are the same set for every seed, in another order."""
    B, nq, nk = c["batch"], c["q_tokens"], c["k_tokens"]
    if not c["ragged"]:
        return [nq] * B, [nk] * B
    most = 3 * c["ring"] + c["sinks"] if c["ring"] else nk
    out = []
    for b in range(B):
        kl = max(1, most - (most * 3 * b) // (4 * B))
        ql = kl if nq == nk and not c["ring"] else max(1, min(nq, kl) - (nq * b) // (2 * B))
        out.append((ql, kl))
    random.Random(seed).shuffle(out)
    return [x[0] for x in out], [x[1] for x in out]


def _views(c, gen, tokens, heads, kv_heads, parts, zero=False):
    """Tensors of shape [B, heads, N, D] as views of the case's memory layout: `parts` gives
    for each whether it has the query or the key/value heads."""
    B, D = c["batch"], c["head_dim"]
    dtype = _DTYPES[c["dtype"]]

    def fill(*shape):
        if zero:
            return torch.zeros(shape, dtype=dtype, device="cuda")
        return torch.randn(shape, generator=gen, device="cuda").to(dtype)

    counts = [heads if p == "q" else kv_heads for p in parts]
    if c["memory"] == "packed":
        buf = fill(B, tokens, sum(counts), D)
        return [t.transpose(1, 2) for t in buf.split(counts, dim=2)]
    if c["memory"] == "tokens":
        return [fill(B, tokens, n, D).transpose(1, 2) for n in counts]
    return [fill(B, n, tokens, D) for n in counts]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c, "op": c["op"]}
    if c["op"].startswith("window"):
        _prepare_window(s, c, gen, seed)
    else:
        _prepare_heads(s, c, gen)
    return s


def _prepare_heads(s, c, gen):
    B, N, D, axes = c["batch"], c["tokens"], c["head_dim"], c["axes"]
    h, kv = c["heads"], c["kv_heads"]
    s["q"], s["k"], s["v"] = _views(c, gen, N, h, kv, "qkk")
    if axes == 2:
        # rows and columns of a grid twice as wide as high
        width = max(1, int(math.sqrt(2.0 * N)))
        t = torch.arange(N, device="cuda")
        s["positions"] = torch.stack([t // width, t % width], dim=-1).to(torch.int32)
    elif c["far"]:
        first = torch.randint(0, c["far"], (B, 1), generator=gen, device="cuda")
        s["positions"] = (first + torch.arange(N, device="cuda")).to(torch.int32).unsqueeze(-1)
    else:
        s["positions"] = torch.arange(N, device="cuda", dtype=torch.int32).unsqueeze(-1)
    if c["op"].startswith("norm"):
        s["qw"] = 1.0 + 0.1 * torch.randn(D, generator=gen, device="cuda")
        s["kw"] = 1.0 + 0.1 * torch.randn(D, generator=gen, device="cuda")
    if c["op"] != "rope_bwd":
        s["q_out"] = torch.empty(B, h, N, D, dtype=s["q"].dtype, device="cuda")
        s["k_out"] = torch.empty(B, kv, N, D, dtype=s["q"].dtype, device="cuda")
    if c["cache"]:
        s["k_out"], s["v_out"] = (
            torch.randn(B, kv, c["cache"], D, generator=gen, device="cuda").to(s["q"].dtype)
            for _ in range(2))
        s["rows"] = torch.randint(0, c["cache"], (B, N), generator=gen,
                                  device="cuda").to(torch.int32)
    if c["op"] in ("rope_bwd", "norm_train"):
        s["dq_out"] = torch.randn(B, h, N, D, generator=gen, device="cuda").to(s["q"].dtype)
        s["dk_out"] = torch.randn(B, kv, N, D, generator=gen, device="cuda").to(s["q"].dtype)
        # gradients go where the projection's backward reads them
        s["dq"], s["dk"], _ = _views(c, gen, N, h, kv, "qkk", zero=True)
    if c["op"] == "norm_train":
        s["dqw"], s["dkw"] = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    if own:
        import paper_2604_16429_amd as bsa
        from paper_2604_16429_amd import binding
        scaling = {"none": binding.SCALE_NONE, "linear": binding.SCALE_LINEAR,
                   "base": binding.SCALE_BASE, "ramp": binding.SCALE_RAMP}[c["scaling"]]
        layout = binding.ROTATE_HALVES if c["layout"] == "halves" else binding.ROTATE_PAIRS
        s["rotation"] = bsa.Rotation(c["rotary_dim"], axes=axes, layout=layout, scaling=scaling,
                                     factor=c["factor"], original_tokens=c["original"])
        s["params"] = bsa.HeadsParams(B, N, h, D, _own_dtype(c), kv_heads=kv,
                                      cache_tokens=c["cache"])
        if c["op"] == "norm_train":
            s["ws"] = torch.empty(bsa.mosaic_bsa_qk_norm_rope_workspace_bytes(s["params"]),
                                  dtype=torch.uint8, device="cuda")


def _own_dtype(c):
    from paper_2604_16429_amd import binding
    return binding.BF16 if c["dtype"] == "bf16" else binding.F32


def _prepare_window(s, c, gen, seed):
    B, D, h, kv = c["batch"], c["head_dim"], c["heads"], c["kv_heads"]
    nq, nk = c["q_tokens"], c["k_tokens"]
    if c["memory"] == "packed":
        s["q"], s["k"], s["v"] = _views(c, gen, nq, h, kv, "qkk")
    else:
        (s["q"],) = _views(c, gen, nq, h, kv, "q")
        s["k"], s["v"] = _views(c, gen, nk, h, kv, "kk")
    # the first tokens draw attention, as such tokens do
    s["k"][:, :, :c["sinks"]] *= 1.5
    s["q_lens"], s["k_lens"] = _lengths(c, seed)
    s["out"] = torch.empty(B, nq, h, D, dtype=s["q"].dtype, device="cuda").transpose(1, 2)
    if c["op"] == "window_train":
        s["dout"] = torch.randn(B, nq, h, D, generator=gen, device="cuda").to(s["q"].dtype)
        s["dout"] = s["dout"].transpose(1, 2)
        if c["memory"] == "packed":
            s["dq"], s["dk"], s["dv"] = _views(c, gen, nq, h, kv, "qkk", zero=True)
        else:
            (s["dq"],) = _views(c, gen, nq, h, kv, "q", zero=True)
            s["dk"], s["dv"] = _views(c, gen, nk, h, kv, "kk", zero=True)
        s["lse"] = torch.empty(B, h, nq, device="cuda")
    if c["ragged"]:
        s["q_lens_d"] = torch.tensor(s["q_lens"], dtype=torch.int32, device="cuda")
        s["k_lens_d"] = torch.tensor(s["k_lens"], dtype=torch.int32, device="cuda")
    if own:
        import paper_2604_16429_amd as bsa
        from paper_2604_16429_amd import binding
        s["params"] = bsa.WindowParams(B, h, nq, nk, D, _own_dtype(c), kv_heads=kv,
                                       window_left=c["left"], window_right=c["right"],
                                       n_sink=c["sinks"], ring=c["ring"])

        def space(op):
            n = bsa.mosaic_bsa_window_workspace_bytes(s["params"], op)
            return torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")

        s["ws"] = space(binding.OP_FWD)
        if c["op"] == "window_train":
            s["ws_b"] = space(binding.OP_BWD)


# ------------------------------------------------------------------ one pass

def run(s):
    if s["op"].startswith("window"):
        return _run_window_own(s) if own else _run_window(s)
    return _run_heads_own(s) if own else _run_heads(s)


def _run_heads_own(s):
    import paper_2604_16429_amd as bsa
    p, r, pos = s["params"], s["rotation"], s["positions"]
    if s["op"] == "rope_fwd":
        bsa.mosaic_bsa_rope_fwd(p, r, pos, s["q"], s["k"], s["q_out"], s["k_out"])
        return s["q_out"], s["k_out"]
    if s["op"] == "rope_bwd":
        bsa.mosaic_bsa_rope_bwd(p, r, pos, s["dq_out"], s["dk_out"], s["dq"], s["dk"])
        return s["dq"], s["dk"]
    if s["case"]["cache"]:
        bsa.mosaic_bsa_qk_norm_rope_fwd(p, r, pos, s["q"], s["k"], s["qw"], s["kw"], s["q_out"],
                                        s["k_out"], v=s["v"], v_out=s["v_out"], rows=s["rows"])
        return s["q_out"], s["k_out"], s["v_out"]
    bsa.mosaic_bsa_qk_norm_rope_fwd(p, r, pos, s["q"], s["k"], s["qw"], s["kw"], s["q_out"],
                                    s["k_out"])
    if s["op"] == "norm_fwd":
        return s["q_out"], s["k_out"]
    bsa.mosaic_bsa_qk_norm_rope_bwd(p, r, pos, s["q"], s["k"], s["qw"], s["kw"], s["dq_out"],
                                    s["dk_out"], s["dq"], s["dk"], s["dqw"], s["dkw"], s["ws"])
    return s["q_out"], s["k_out"], s["dq"], s["dk"], s["dqw"], s["dkw"]


def _run_window_own(s):
    import paper_2604_16429_amd as bsa
    p, lens = s["params"], dict(q_lens=s.get("q_lens_d"), k_lens=s.get("k_lens_d"))
    bsa.mosaic_bsa_window_fwd(p, s["q"], s["k"], s["v"], s["out"], s.get("lse"),
                              workspace=s["ws"], **lens)
    if s["op"] == "window_fwd":
        return s["out"]
    bsa.mosaic_bsa_window_bwd(p, s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["dq"],
                              s["dk"], s["dv"], s["ws_b"], **lens)
    return s["out"], s["dq"], s["dk"], s["dv"]


# ---- plain form: rotation and norms

_THETA = 10000.0
_BETA_FAST, _BETA_SLOW = 32.0, 1.0
_EPS = 1e-6


def _frequencies(c, device):
    """(angle per position of each pair of one axis in 64 bits, magnitude)."""
    d = c["rotary_dim"] // c["axes"]
    e = torch.arange(d // 2, device=device, dtype=torch.float64) * 2.0 / d
    theta, f, mag = _THETA, c["factor"], 1.0
    if c["scaling"] == "base":
        theta = theta * f ** (d / (d - 2.0))
    w = torch.exp(-math.log(theta) * e)
    if c["scaling"] == "linear":
        w = w / f
    if c["scaling"] == "ramp":
        turns = c["original"] * w / (2.0 * math.pi)
        keep = ((turns - _BETA_SLOW) / (_BETA_FAST - _BETA_SLOW)).clamp(0.0, 1.0)
        w = keep * w + (1.0 - keep) * w / f
        mag = 0.1 * math.log(f) + 1.0
    return w, mag


def _cos_sin(c, positions):
    """[B or 1, 1, N, axes * pairs] cosines and sines, fp32 from angles in 64 bits."""
    w, mag = _frequencies(c, positions.device)
    angle = positions.double().unsqueeze(-1) * w              # [.., N, axes, pairs]
    angle = angle.flatten(-2)
    if angle.dim() == 2:
        angle = angle.unsqueeze(0)
    angle = angle.unsqueeze(1)
    return (torch.cos(angle) * mag).float(), (torch.sin(angle) * mag).float()


def _rotated(c, x, cos, sin):
    """Rotation of fp32 [B, heads, N, D]; sin negated: its transpose."""
    rd, axes = c["rotary_dim"], c["axes"]
    p = rd // axes // 2
    head = x[..., :rd]
    shape = head.shape[:-1]
    if c["layout"] == "halves":
        a, b = head.reshape(*shape, axes, 2, p).unbind(-2)
    else:
        a, b = head.reshape(*shape, axes, p, 2).unbind(-1)
    a, b = a.flatten(-2), b.flatten(-2)
    u = (a * cos - b * sin).view(*shape, axes, p)
    v = (b * cos + a * sin).view(*shape, axes, p)
    turned = torch.stack([u, v], dim=-2 if c["layout"] == "halves" else -1).reshape(*shape, rd)
    return torch.cat([turned, x[..., rd:]], dim=-1) if rd < x.shape[-1] else turned


def _run_heads(s):
    c = s["case"]
    cos, sin = _cos_sin(c, s["positions"])
    dtype = s["q"].dtype
    if s["op"] == "rope_fwd":
        return tuple(_rotated(c, s[t].float(), cos, sin).to(dtype) for t in "qk")
    if s["op"] == "rope_bwd":
        return tuple(_rotated(c, s[t].float(), cos, -sin).to(dtype) for t in ("dq_out", "dk_out"))
    out, grads, weight_grads = [], [], []
    for t in "qk":
        x, g = s[t].float(), s[t + "w"]
        r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + _EPS)
        n = x * r
        out.append(_rotated(c, n * g, cos, sin).to(dtype))
        if s["op"] == "norm_train":
            dz = _rotated(c, s["d" + t + "_out"].float(), cos, -sin)
            # a sum over all rows: in 64 bits
            weight_grads.append((dz * n).sum(dim=(0, 1, 2), dtype=torch.float64).float())
            dn = dz * g
            grads.append((r * (dn - n * (dn * n).mean(dim=-1, keepdim=True))).to(dtype))
    if c["cache"]:
        rows = s["rows"].long()
        b = torch.arange(c["batch"], device=rows.device).unsqueeze(1)
        s["k_out"][b, :, rows] = out[1].transpose(1, 2)
        s["v_out"][b, :, rows] = s["v"].transpose(1, 2)
        return out[0], s["k_out"], s["v_out"]
    return tuple(out + grads + weight_grads)


# ---- plain form: windowed attention

_CHUNK = 256           # query tokens of a plain pass at a time


def _key_range(c, first, last, length):
    """Tokens lo .. hi that queries at positions first .. last can see beside the sinks."""
    hi = length - 1 if c["right"] < 0 else min(length - 1, last + c["right"])
    lo = 0 if c["left"] < 0 else max(0, first - c["left"])
    return lo, hi


def _sequences(s):
    """(slice of the batch, query length, key length): whole batches of one length at once."""
    c = s["case"]
    if not c["ragged"]:
        return [(slice(0, c["batch"]), c["q_tokens"], c["k_tokens"])]
    return [(slice(b, b + 1), s["q_lens"][b], s["k_lens"][b]) for b in range(c["batch"])]


def _run_window(s):
    c = s["case"]
    q, k, v = s["q"], s["k"], s["v"]
    train = s["op"] == "window_train"
    B, h, nq, D = q.shape
    kv, G = c["kv_heads"], c["heads"] // c["kv_heads"]
    scale = 1.0 / math.sqrt(D)
    dev = q.device
    out = torch.zeros(B, h, nq, D, device=dev)
    if train:
        dq, dk, dv = (torch.zeros(t.shape, device=dev) for t in (q, k, v))
    for sl, ql, kl in _sequences(s):
        for q0 in range(0, ql, _CHUNK):
            q1 = min(ql, q0 + _CHUNK)
            p0 = kl - ql
            lo, hi = _key_range(c, p0 + q0, p0 + q1 - 1, kl)
            ns = max(0, min(c["sinks"], lo, hi + 1))
            tok = torch.cat([torch.arange(ns, device=dev), torch.arange(lo, hi + 1, device=dev)])
            row = tok
            if c["ring"]:
                row = torch.where(tok < c["sinks"], tok,
                                  c["sinks"] + (tok - c["sinks"]) % c["ring"])
            n = q1 - q0
            b = sl.stop - sl.start
            qc = q[sl, :, q0:q1].float().reshape(b * kv, G * n, D)
            kc = k[sl][:, :, row].float().reshape(b * kv, -1, D)
            vc = v[sl][:, :, row].float().reshape(b * kv, -1, D)
            pos = p0 + torch.arange(q0, q1, device=dev).unsqueeze(1)
            seen = torch.ones(n, tok.numel(), dtype=torch.bool, device=dev)
            if c["right"] >= 0:
                seen &= tok <= pos + c["right"]
            if c["left"] >= 0:
                seen &= (tok >= pos - c["left"]) | (tok < c["sinks"])
            seen = seen.repeat(G, 1)
            x = torch.matmul(qc, kc.transpose(1, 2)) * scale
            x = x.masked_fill(~seen, -math.inf)
            top = x.amax(dim=-1, keepdim=True)
            top = torch.where(top == -math.inf, torch.zeros_like(top), top)
            w = torch.exp(x - top)
            total = w.sum(dim=-1, keepdim=True)
            w = w / torch.where(total > 0.0, total, torch.ones_like(total))
            o = torch.matmul(w, vc)
            out[sl, :, q0:q1] = o.view(b, h, n, D)
            if train:
                do = s["dout"][sl, :, q0:q1].float().reshape(b * kv, G * n, D)
                dv_c = torch.matmul(w.transpose(1, 2), do)
                dx = w * (torch.matmul(do, vc.transpose(1, 2)) -
                          (do * o).sum(dim=-1, keepdim=True)) * scale
                dq[sl, :, q0:q1] = torch.matmul(dx, kc).view(b, h, n, D)
                dk_c = torch.matmul(dx.transpose(1, 2), qc)
                for grad, part in ((dk, dk_c), (dv, dv_c)):
                    part = part.view(b, kv, -1, D)
                    grad[sl, :, :ns] += part[:, :, :ns]
                    grad[sl, :, lo:hi + 1] += part[:, :, ns:]
    out = out.to(q.dtype)
    if not train:
        return out
    return out, dq.to(q.dtype), dk.to(q.dtype), dv.to(q.dtype)


# ------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"].startswith("window"):
        return _exact_window(s, c)
    return _exact_heads(s, c)


def _exact_turn(c, x, positions, sign):
    """x as complex numbers times exp(i sign position w): fp64 [B, heads, N, D]."""
    rd, axes = c["rotary_dim"], c["axes"]
    d = rd // axes
    f = c["factor"]
    base = 10000.0 * (f ** (d / (d - 2)) if c["scaling"] == "base" else 1.0)
    ws, mag = [], 1.0
    for i in range(d // 2):
        w = base ** (-2.0 * i / d)
        if c["scaling"] == "linear":
            w /= f
        elif c["scaling"] == "ramp":
            r = c["original"] * w / (2.0 * math.pi)
            g = 0.0 if r < 1.0 else 1.0 if r > 32.0 else (r - 1.0) / 31.0
            w = (1.0 - g) * w / f + g * w
            mag = 0.1 * math.log(f) + 1.0
        ws.append(w)
    w = torch.tensor(ws, dtype=torch.float64, device=x.device)
    pos = positions if positions.dim() == 3 else positions.unsqueeze(0)
    parts = []
    for a in range(axes):
        y = x[..., a * d:(a + 1) * d]
        even, odd = ((y[..., :d // 2], y[..., d // 2:]) if c["layout"] == "halves"
                     else (y[..., 0::2], y[..., 1::2]))
        phase = sign * pos[..., a].double()[:, None, :, None] * w
        z = torch.complex(even.contiguous(), odd.contiguous()) * torch.polar(
            torch.full_like(phase, mag), phase)
        y = (torch.cat([z.real, z.imag], -1) if c["layout"] == "halves"
             else torch.view_as_real(z).flatten(-2))
        parts.append(y)
    return torch.cat(parts + [x[..., rd:]], -1)


def _exact_heads(s, c):
    pos = s["positions"]
    if c["op"] == "rope_fwd":
        return tuple(_exact_turn(c, s[t].double(), pos, 1.0) for t in "qk")
    if c["op"] == "rope_bwd":
        return tuple(_exact_turn(c, s["d" + t + "_out"].double(), pos, -1.0) for t in "qk")
    outs, grads, weight_grads = [], [], []
    train = c["op"] == "norm_train"
    for t in "qk":
        x = s[t].double().requires_grad_(train)
        g = s[t + "w"].double().requires_grad_(train)
        y = _exact_turn(c, g * x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6), pos, 1.0)
        if train:
            dx, dg = torch.autograd.grad(y, (x, g), s["d" + t + "_out"].double())
            grads.append(dx)
            weight_grads.append(dg)
        outs.append(y.detach())
    if c["cache"]:
        k_out, v_out = s["k_out"].double(), s["v_out"].double()
        for b in range(c["batch"]):
            for n in range(c["tokens"]):
                r = int(s["rows"][b, n])
                k_out[b, :, r] = outs[1][b, :, n]
                v_out[b, :, r] = s["v"][b, :, n].double()
        return outs[0], k_out, v_out
    return tuple(outs + grads + weight_grads)


def _exact_window(s, c):
    train = c["op"] == "window_train"
    q, k, v = s["q"], s["k"], s["v"]
    B, h, nq, D = q.shape
    G = h // c["kv_heads"]
    out = torch.zeros(B, h, nq, D, dtype=torch.float64, device=q.device)
    if train:
        dq, dk, dv = (torch.zeros(t.shape, dtype=torch.float64, device=q.device)
                      for t in (q, k, v))
    step = 512
    for b in range(B):
        ql, kl = s["q_lens"][b], s["k_lens"][b]
        for a in range(c["kv_heads"]):
            heads = slice(a * G, (a + 1) * G)
            for i0 in range(0, ql, step):
                i1 = min(i0 + step, ql)
                p = torch.arange(kl - ql + i0, kl - ql + i1, device=q.device)
                end = kl if c["right"] < 0 else min(kl, int(p[-1]) + c["right"] + 1)
                beg = 0 if c["left"] < 0 else max(0, int(p[0]) - c["left"])
                j = torch.arange(end, device=q.device)
                j = j[(j < c["sinks"]) | (j >= beg)]
                where = j
                if c["ring"]:
                    where = j.clone()
                    late = j >= c["sinks"]
                    where[late] = (j[late] - c["sinks"]) % c["ring"] + c["sinks"]
                x = q[b, heads, i0:i1].double().requires_grad_(train)
                y = k[b, a, where].double().requires_grad_(train)
                z = v[b, a, where].double().requires_grad_(train)
                d = p[:, None] - j[None, :]
                hidden = torch.zeros_like(d, dtype=torch.bool)
                if c["right"] >= 0:
                    hidden |= d < -c["right"]
                if c["left"] >= 0:
                    hidden |= (d > c["left"]) & (j >= c["sinks"])[None, :]
                # rows that see nothing: zeros
                none = hidden.all(dim=1)
                logits = (x @ y.t()) / math.sqrt(D)
                logits = logits.masked_fill(hidden & ~none[:, None], -math.inf)
                o = torch.softmax(logits, dim=-1).masked_fill(none[:, None], 0.0) @ z
                out[b, heads, i0:i1] = o.detach()
                if train:
                    gx, gy, gz = torch.autograd.grad(
                        o, (x, y, z), s["dout"][b, heads, i0:i1].double())
                    dq[b, heads, i0:i1] = gx
                    dk[b, a].index_add_(0, j, gy)
                    dv[b, a].index_add_(0, j, gz)
    return (out, dq, dk, dv) if train else out


# ------------------------------------------------------------------ work

def work(case):
    c = case
    esz = 2 if c["dtype"] == "bf16" else 4
    return _work_window(c, esz) if c["op"].startswith("window") else _work_heads(c, esz)


def _work_heads(c, esz):
    rows = c["batch"] * c["tokens"] * (c["heads"] + c["kv_heads"])
    tensor = rows * c["head_dim"] * esz
    rotate = 3.0 * rows * c["rotary_dim"]                # two products and a sum per value
    position = 4 * c["tokens"] * c["axes"] * (c["batch"] if c["far"] else 1)
    nbytes, flops = 2 * tensor + position, rotate
    if c["op"].startswith("norm"):
        flops += 4.0 * rows * c["head_dim"]              # square, sum, two products
        nbytes += 8 * c["head_dim"]
    if c["cache"]:
        nbytes += 2 * c["batch"] * c["tokens"] * c["kv_heads"] * c["head_dim"] * esz
    if c["op"] == "norm_train":
        # gradients and inputs in, gradients out
        nbytes += 3 * tensor + position + 16 * c["head_dim"]
        flops += rotate + 12.0 * rows * c["head_dim"]
    return {"bytes": float(nbytes), "flops": float(flops)}


def _work_window(c, esz):
    pairs, keys, queries = 0, 0, 0
    for ql, kl in zip(*_lengths(c, 0)):
        p = torch.arange(kl - ql, kl, dtype=torch.int64)
        p = p[p >= 0] if c["right"] == 0 else p
        hi = torch.full_like(p, kl - 1) if c["right"] < 0 else (p + c["right"]).clamp(max=kl - 1)
        lo = torch.zeros_like(p) if c["left"] < 0 else (p - c["left"]).clamp(min=0)
        sink = torch.minimum(lo, hi + 1).clamp(min=0, max=c["sinks"])
        pairs += int((hi - lo + 1).clamp(min=0).sum() + sink.sum())
        queries += ql
        if p.numel():
            first = int(lo.min())
            keys += int(hi.max()) - first + 1 + min(c["sinks"], first)
    D, h, kv = c["head_dim"], c["heads"], c["kv_heads"]
    q_bytes, kv_bytes = queries * h * D * esz, 2 * keys * kv * D * esz
    nbytes = 2 * q_bytes + kv_bytes
    flops = 4.0 * pairs * h * D
    if c["op"] == "window_train":
        # dout in, dq, dk, dv out; five products for two
        nbytes += 2 * q_bytes + kv_bytes
        flops += 10.0 * pairs * h * D
    return {"bytes": float(nbytes), "flops": float(flops)}
