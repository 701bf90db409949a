"""Plain 64-bit attention of packed prompts with its gradient, from the formulas, and the
bounds that the kernels' results are held to."""

from __future__ import annotations

import math

import torch

from cache_reference import TINY, UNIT


def attend(q, k, v, row_off, key_off=None, scale=0.0, causal=True):
    """(out, lse, bound of out without its last rounding, bound of lse) in float64, on q's device.

    The bounds. A score's error is at most (dim + 8) fp32 roundings of the sum of its
    terms' magnitudes (tensor cores may truncate: twice that), and the exponential's 2^-20: d. A
    probability is rounded to the values' type (f16: 2^-32 of the largest may be lost besides). Sums of m keys
    are added 16 at a time in fp32.
    """
    u, f64 = UNIT[q.dtype], torch.float64
    key_off = row_off if key_off is None else key_off
    rows, H, D = q.shape
    G = H // k.shape[1]
    scale = scale or 1.0 / math.sqrt(D)
    out = torch.zeros((rows, H, D), dtype=f64, device=q.device)
    lse = torch.full((rows, H), -math.inf, dtype=f64, device=q.device)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    for i in range(len(row_off) - 1):
        a, b = slice(row_off[i], row_off[i + 1]), slice(key_off[i], key_off[i + 1])
        r, m = a.stop - a.start, b.stop - b.start
        if r == 0 or m == 0:
            continue
        see = torch.ones((r, m), dtype=torch.bool, device=q.device)
        if causal:
            see = see.tril(m - r)
        add = (m / 8 + 16) * 2.0 ** -23
        for h in range(H):
            Q, K, V = q[a, h].double(), k[b, h // G].double(), v[b, h // G].double()
            x = torch.where(see, (Q @ K.T) * scale, -math.inf)
            top = x.amax(-1, keepdim=True)
            top = torch.where(top == -math.inf, 0.0, top)
            p = torch.exp(x - top)
            l = p.sum(-1, keepdim=True)
            p = torch.where(l > 0, p / l, p)
            odd = ~torch.isfinite(V)
            Vz = torch.where(odd, 0.0, V)
            o = p @ Vz
            for bad, y in ((torch.isnan(V), math.nan), (V == math.inf, math.inf), (V == -math.inf, -math.inf)):
                o = o + torch.where(see.double() @ bad.double() > 0, y, 0.0)
            out[a, h] = o
            lse[a, h] = (top + torch.log(l))[:, 0]
            mass = (Q.abs() @ K.abs().T * scale).nan_to_num(0, 0, 0).amax(-1, keepdim=True)
            d = (D + 8) * 2.0 ** -23 * mass + 2.0 ** -20
            lost = (2.0 ** -31 if q.dtype == torch.float16 else 2.0 ** -90) * (see.double() @ Vz.abs()) / l.clamp(min=1.0)
            out_tol[a, h] = (u + 2 * d + add) * (p.nan_to_num() @ Vz.abs()) + lost
            lse_tol[a, h] = d[:, 0] + add + 2.0 ** -20 + 2.0 ** -22 * lse[a, h].nan_to_num(0, 0, 0).abs()
    return out, lse, out_tol, lse_tol


def assert_near(got, want, tol, dtype, where=""):
    """|got - want| <= tol and got's own rounding; what is not finite has to be the same."""
    g = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(g), torch.isnan(want)), f"{where}: NaN differs"
    assert torch.equal(g[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), f"{where}: infinities differ"
    off = (g - want).abs() - (tol + UNIT[dtype] * (want.abs() + tol) + TINY[dtype])
    off = torch.where(fine, off, -1.0)
    assert off.numel() == 0 or float(off.max()) <= 0, f"{where}: {float(off.max())} past its bound at {divmod(int(off.argmax()), got.shape[-1])}"


def grad(q, k, v, dout, row_off, key_off=None, scale=0.0, causal=True):
    """(dq, dk, dv and the bounds of each without its last rounding) in float64, from the formulas.

    The bounds. p is exp of a score less lse, both off (d and attend()'s bound of lse): e; it is rounded to the
    inputs' type (u; f16: held 2^14 times as large, 2^-39 may be lost) for dv. ds = p (dP - delta): dP is a sum of dim fp32
    products, delta comes from an out that is off and rounded; ds is rounded (f16: within 2^-25 of 2^14
    times what is at least a quarter of its bound |dO||V| + |delta|, so 2^-37 of that may be lost). Sums are in fp32, 16 terms at
    a time.
    """
    u, f64, f16 = UNIT[q.dtype], torch.float64, q.dtype == torch.float16
    key_off = row_off if key_off is None else key_off
    rows, H, D = q.shape
    G = H // k.shape[1]
    sc = scale or 1.0 / math.sqrt(D)
    out, lse, out_tol, lse_tol = attend(q, k, v, row_off, key_off, scale, causal)
    res = [torch.zeros(x.shape, dtype=f64, device=q.device) for x in (q, k, v)]
    tol = [torch.zeros_like(x) for x in res]
    for i in range(len(row_off) - 1):
        a, b = slice(row_off[i], row_off[i + 1]), slice(key_off[i], key_off[i + 1])
        r, m = a.stop - a.start, b.stop - b.start
        if r == 0 or m == 0:
            continue
        see = torch.ones((r, m), dtype=torch.bool, device=q.device)
        if causal:
            see = see.tril(m - r)
        add = (r * G / 8 + m / 8 + 32) * 2.0 ** -23
        for h in range(H):
            Q, K, V, dO = q[a, h].double(), k[b, h // G].double(), v[b, h // G].double(), dout[a, h].double()
            O, L = out[a, h], lse[a, h][:, None]
            p = torch.where(see, torch.exp((Q @ K.T) * sc - torch.where(L == -math.inf, 0.0, L)), 0.0)
            delta = (dO * O).sum(-1, keepdim=True)
            g = torch.where(see, dO @ V.T - delta, 0.0)
            ds = p * g
            res[0][a, h] = sc * (ds @ K)
            res[1][b, h // G] += sc * (ds.T @ Q)
            res[2][b, h // G] += p.T @ dO
            mass = (Q.abs() @ K.abs().T * sc).amax(-1, keepdim=True)
            e = 2 * ((D + 8) * 2.0 ** -23 * mass + 2.0 ** -20 + lse_tol[a, h][:, None] + 2.0 ** -22 * torch.where(L == -math.inf, 0.0, L).abs())
            p_err = torch.where(see, p * (u + e) + (2.0 ** -39 if f16 else 0.0), 0.0)
            dp_err = (D + 8) * 2.0 ** -23 * (dO.abs() @ V.abs().T)
            delta_err = (dO.abs() * (u * O.abs() + (1 + u) * out_tol[a, h])).sum(-1, keepdim=True) + (D + 8) * 2.0 ** -24 * (dO * O).abs().sum(-1, keepdim=True)
            bound = dO.norm(dim=-1).max() * V.norm(dim=-1).max() + delta.abs().max()
            # (the group's other heads share the power of two: at most the largest of their bounds)
            for h2 in range(h // G * G, h // G * G + G) if f16 else ():
                d2 = dout[a, h2].double()
                bound = torch.maximum(bound, d2.norm(dim=-1).max() * V.norm(dim=-1).max() + (d2 * out[a, h2]).sum(-1).abs().max())
            ds_err = torch.where(see, p * ((u + 2 * e) * g.abs() + (1 + u) * (dp_err + delta_err)) + (2.0 ** -36 * bound if f16 else 0.0), 0.0)
            tol[0][a, h] = sc * (ds_err @ K.abs()) + add * sc * (ds.abs() @ K.abs())
            tol[1][b, h // G] += sc * (ds_err.T @ Q.abs()) + add * sc * (ds.abs().T @ Q.abs())
            tol[2][b, h // G] += p_err.T @ dO.abs() + add * (p.T @ dO.abs())
    return (*res, *tol)
