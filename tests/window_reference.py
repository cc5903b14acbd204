"""Windowed attention, rotation and head norms written out in 64 bits on the CPU, with bounds
on what the kernels' roundings may change; shares no code with the package."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def visible(ql, kl, nq, nk, left, right, sinks):
    """[nq, nk] truth values for one sequence; rows past ql and keys past kl see nothing."""
    i = torch.arange(nq).unsqueeze(1)
    j = torch.arange(nk).unsqueeze(0)
    p = kl - ql + i
    see = (i < ql) & (j < kl)
    if right >= 0:
        see = see & (j <= p + right)
    if left >= 0:
        see = see & ((j >= p - left) | (j < sinks))
    return see


def attention(q, k, v, see, scale, dout=None):
    """One (batch, head): q [nq, D], k, v [nk, D] in 64 bits, see [nq, nk].  Returns a dict of
    results (out, lse; dq, dk, dv with dout) and of the bounds, "<name>_tol" as functions of
    the element type, on the distance of a computation that holds scores, sums and statistics
    in 32 bits and rounds weights, score gradients and outputs to the element type."""
    k = torch.where(see.any(0).unsqueeze(1), k, torch.zeros_like(k))     # (may hold anything)
    v = torch.where(see.any(0).unsqueeze(1), v, torch.zeros_like(v))
    s = (q @ k.T) * scale
    s = s.masked_fill(~see, -math.inf)
    lse = torch.logsumexp(s, dim=1)
    none = ~see.any(1)
    p = torch.exp(s - torch.where(none, torch.zeros_like(lse), lse).unsqueeze(1))
    p = p.masked_fill(~see, 0.0)
    out = p @ v
    r = {"out": out, "lse": lse}
    D, n = q.shape[1], k.shape[0]
    u32 = 2.0 ** -24
    # a score is a sum of D products in 32 bits, its exponential good to 2^-21
    size = (q.abs() @ k.abs().T) * scale
    w_rel = 2.0 * (D + 4) * u32 * float(size.max()) + 2.0 ** -21 + 2.0 * (n + 8) * u32

    def half(dtype):
        # what rounding a weight to the operand type may change, beside w_rel
        return 0.0 if dtype is torch.float32 else HALF_STEP[dtype]

    def out_tol(dtype):
        return ((p @ v.abs()) * (half(dtype) + w_rel) + out.abs() * HALF_STEP[dtype]) * 1.01 + 1e-30

    r["out_tol"] = out_tol
    r["lse_tol"] = w_rel + 2.0 ** -22 * lse.abs()
    if dout is None:
        return r
    g = dout
    dp = g @ v.T
    delta = (g * out).sum(1, keepdim=True)
    ds = p * (dp - delta)
    r["dv"], r["dq"], r["dk"] = p.T @ g, (ds @ k) * scale, (ds.T @ q) * scale

    def grad_tol(name):
        def tol(dtype):
            h = half(dtype)
            # delta comes from the rounded output
            d_delta = (g.abs() * out_tol(dtype)).sum(1, keepdim=True) + \
                (D + 2) * u32 * (g.abs() * out.abs()).sum(1, keepdim=True)
            d_dp = (D + 2) * u32 * (g.abs() @ v.abs().T)
            ds_err = ds.abs() * (h + w_rel) + p * (d_delta + d_dp) * (1.0 + h)
            sums = 2.0 * (n + q.shape[0]) * u32
            if name == "dv":
                e = (p * (h + w_rel + sums)).T @ g.abs()
            elif name == "dq":
                e = ((ds_err + sums * ds.abs()) @ k.abs()) * scale
            else:
                e = ((ds_err + sums * ds.abs()).T @ q.abs()) * scale
            # dk and dv of a group's heads are added in 32 bits and rounded once: the caller
            # adds the rounding of the sum
            return e * 1.01 + 1e-30
        return tol

    for name in ("dq", "dk", "dv"):
        r[name + "_tol"] = grad_tol(name)
    return r


def rotate(x, positions, inv_freq, magnitude, rotary_dim, axes, pairs, transpose=False):
    """x [B, h, N, D] in 64 bits, positions [B or 1, N, axes] whole numbers, inv_freq [d / 2]."""
    d = rotary_dim // axes
    out = x.clone()
    for a in range(axes):
        for i in range(d // 2):
            c0, c1 = (a * d + 2 * i, a * d + 2 * i + 1) if pairs else (a * d + i, a * d + i + d // 2)
            t = positions[..., a].double() * inv_freq[i]
            cos, sin = torch.cos(t).unsqueeze(1) * magnitude, torch.sin(t).unsqueeze(1) * magnitude
            if transpose:
                sin = -sin
            out[..., c0] = x[..., c0] * cos - x[..., c1] * sin
            out[..., c1] = x[..., c1] * cos + x[..., c0] * sin
    return out
