"""Bounds on the windowed attention's bf16 gradients that count each rounding of the kernels once:
delta is a sum of weights times dP in 32 bits, so that the rounding of the output has no part in dQ and
dK but in the second order.  Results come from window_reference.attention."""
import math

import torch

from tests.window_reference import HALF_STEP, attention

U32 = 2.0 ** -24


def attention_and_bounds(q, k, v, see, scale, g, group=1):
    """As attention, with "dq_tol", "dk_tol" and "dv_tol" as tensors for bf16 (before the rounding of the
    result, which the caller adds).  group: heads whose sums dk and dv are."""
    r = attention(q, k, v, see, scale, g)
    seen = see.any(0).unsqueeze(1)
    k, v = (torch.where(seen, t, torch.zeros_like(t)) for t in (k, v))
    h, (nq, D), n = HALF_STEP[torch.bfloat16], q.shape, k.shape[0]
    none = ~see.any(1)
    lse = torch.where(none, torch.zeros_like(r["lse"]), r["lse"])
    p = torch.exp((q @ k.T) * scale - lse.unsqueeze(1)).masked_fill(~see, 0.0)
    size = float(((q.abs() @ k.abs().T) * scale).max())
    # a weight: its score, D products in 32 bits; lse, a score of the same size and a sum of n weights, held in
    # 32 bits in one base and the other; exponential and logarithm to 2^-21
    w_rel = 2.0 * (D + 8) * U32 * size + 2.0 ** -20 + 2.0 * (n + 16) * U32
    # dP - delta: D products, added to delta
    a = g.abs() @ v.abs().T
    d_dp = 2.0 * (D + 4) * U32 * (a + a.amax(1, keepdim=True))
    d_delta = (p * ((w_rel + 2.0 * (n + 4) * U32) * a + d_dp)).sum(1, keepdim=True)
    # the general kernels take delta of the rounded output first and correct their sums by e, the sum of
    # dS, with weights rounded like dS
    e = (g.abs() * r["out_tol"](torch.bfloat16)).sum(1, keepdim=True) + d_delta
    ds = p * ((g @ v.T) - (g * r["out"]).sum(1, keepdim=True))
    sums = 2.0 * (n + group * nq + 64) * U32
    ds_err = ds.abs() * (h + w_rel + sums) + p * (d_delta + d_dp) * (1.0 + h + w_rel) + \
        p * e * (2.0 * h + w_rel + sums)
    r["dq_tol"] = (ds_err @ k.abs()) * scale * 1.01 + 1e-30
    r["dk_tol"] = (ds_err.T @ q.abs()) * scale * 1.01 + 1e-30
    r["dv_tol"] = (p * (h + w_rel + sums)).T @ g.abs() * 1.01 + 1e-30
    return r


def check_training(got, q, k, v, g, kv, see_of, scale=0.0):
    """got: dict of out, lse, dq, dk, dv, [B, heads, N, D] in 64 bits, of bf16 tensors q, k, v, g in 64
    bits; see_of(b): who sees whom.  Returns the worst share of each bound."""
    B, heads, nq, D = q.shape
    G = heads // kv
    h = HALF_STEP[torch.bfloat16]
    sc = scale if scale > 0.0 else 1.0 / math.sqrt(D)
    worst = {}

    def close(name, x, ref, tol):
        d = (x - ref).abs()
        share = torch.where(x == ref, torch.zeros_like(d), d / tol)
        worst[name] = max(worst.get(name, 0.0), float(share.max()))
        assert bool((share <= 1.0).all()), f"{name}: {float(share.max())} of the bound"

    for b in range(B):
        see = see_of(b)
        alive = see.any(1).unsqueeze(1)
        for a in range(kv):
            sums = {name: [0.0, 0.0] for name in ("dk", "dv")}
            for i in range(a * G, (a + 1) * G):
                qq, gg = (torch.where(alive, t[b, i], torch.zeros_like(t[b, i])) for t in (q, g))
                r = attention_and_bounds(qq, k[b, a], v[b, a], see, sc, gg, G)
                close("out", got["out"][b, i], r["out"], r["out_tol"](torch.bfloat16))
                close("lse", got["lse"][b, i], r["lse"], r["lse_tol"])
                close("dq", got["dq"][b, i], r["dq"], r["dq_tol"] + r["dq"].abs() * h)
                for name, s in sums.items():
                    s[0], s[1] = s[0] + r[name], s[1] + r[name + "_tol"]
            for name, (ref, tol) in sums.items():
                close(name, got[name][b, a], ref, tol + ref.abs() * h)
    return worst
