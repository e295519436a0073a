"""Chunks of new tokens in float64, straight from the definition in include/dynts.h, with bounds on what the kernels may be off.

A product of d terms in fp32 is off by (d + 8) half steps of 2^-24 of the sum of its terms' sizes at most; scaling, capping, the bias and
the shift add a few half steps of the logit's, the cap's and the bias's size.  Those make a weight relatively as much off.
Rounding a weight to bf16 for its product with V, and the output, half a step each: 2^-8.  A weight below the smallest normal fp32 number,
2^-126, is 0: 2^-126 a row on top of what a slot receives."""
import math

import torch

HALF16, HALF32 = 2.0 ** -8, 2.0 ** -24


def attention(q, K, V, pos, n, m, scale, softcap=0.0, window=0, slope=None, first=None, last=None, device="cpu"):
    """One sequence: q [T][Hq][d], K, V [Hkv][>= n][d], pos [Hkv][>= n]; its last m tokens are the queries.
    -> dict of out [m][Hq][d], lse [m][Hq], recv [Hkv][n] and bounds out_tol, lse_tol, recv_tol."""
    Hq, d = q.shape[1:]
    Hkv = K.shape[0]
    G = Hq // Hkv
    q, K, V = (x.to(device, torch.float64) for x in (q[:m], K[:, :n], V[:, :n]))
    pos = pos[:, :n].to(device, torch.int64)
    r = dict(out=torch.zeros(m, Hq, d, dtype=torch.float64), lse=torch.zeros(m, Hq, dtype=torch.float64),
             recv=torch.zeros(Hkv, n, dtype=torch.float64))
    r = {k: x.to(device) for k, x in r.items()}
    r.update(out_tol=torch.zeros_like(r["out"]), lse_tol=torch.zeros_like(r["lse"]), recv_tol=torch.zeros_like(r["recv"]))
    for hq in range(Hq):
        h = hq // G
        x = (q[:, hq] @ K[h].t()) * scale
        size = (q[:, hq].abs() @ K[h].abs().t()) * scale
        off = (d + 8) * HALF32 * size + 8 * HALF32 * x.abs()
        own = pos[h, n - m:n]
        if softcap > 0:
            x = softcap * torch.tanh(x / softcap)
            off = off + 8 * HALF32 * softcap
        if slope is not None:
            bias = float(slope[hq]) * (own[:, None] - pos[h][None]).abs().double()
            x = x - bias
            off = off + 8 * HALF32 * bias
        shaped = softcap > 0 or window > 0 or slope is not None or first is not None or last is not None
        if shaped:
            high = own if last is None else last[:m].to(device, torch.int64)
            low = torch.full_like(own, -1)
            if window > 0:
                low = own - window + 1
            if first is not None:
                low = torch.maximum(low, first[:m].to(device, torch.int64))
            seen = (pos[h][None] >= low[:, None]) & (pos[h][None] <= high[:, None])
        else:
            seen = torch.arange(n, device=device)[None] <= (n - m + torch.arange(m, device=device))[:, None]
        x = torch.where(seen, x, -math.inf)
        off = torch.where(seen, off, 0.0)
        lse = torch.logsumexp(x, dim=-1)
        some = torch.isfinite(lse)
        w = torch.where(seen & some[:, None], torch.exp(x - torch.where(some, lse, 0.0)[:, None]), 0.0)
        # (in log2 units numbers are larger by log2 e < 1.5: their half steps too)
        lse_tol = 1.5 * ((w * off).sum(-1) + (n + 8) * HALF32) + 8 * HALF32 * torch.where(some, lse, 0.0).abs()
        rel = 1.5 * off + lse_tol[:, None] + 8 * HALF32 * (torch.where(seen, x, 0.0).abs() + torch.where(some, lse, 0.0).abs()[:, None])
        spread = w @ V[h].abs()
        r["out"][:, hq] = w @ V[h]
        r["out_tol"][:, hq] = HALF16 * (spread + r["out"][:, hq].abs()) * (1 + HALF16) + (w * 2 * rel) @ V[h].abs() + n * HALF32 * spread
        r["lse"][:, hq], r["lse_tol"][:, hq] = lse, lse_tol
        r["recv"][h] += w.sum(0)
        r["recv_tol"][h] += (w * (torch.exp(rel) - 1)).sum(0) + (m * G + 8) * HALF32 * w.sum(0) + m * 2.0 ** -126
    return {k: x.cpu() for k, x in r.items()}


def check(got, ref, tol, what):
    """Both non-finite alike, and within tol elsewhere; returns the worst share of tol that is used."""
    got, ref = got.detach().double().cpu(), ref
    fin = torch.isfinite(ref)
    assert torch.equal(got[~fin], ref[~fin]), "%s: non-finite entries differ" % what
    off = (got[fin] - ref[fin]).abs()
    bad = ~(off <= tol[fin])
    assert not bad.any(), "%s: %d of %d outside, worst %.3e of %.3e" % (
        what, int(bad.sum()), bad.numel(), float(off[bad].max()), float(tol[fin][bad].max()))
    return float((off / tol[fin].clamp(min=1e-300)).max()) if off.numel() else 0.0
