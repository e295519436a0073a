"""Caches of 8-bit codes and drafts that branch, in float64 straight from the definitions in include/dynts.h."""
import math

import torch

from tests import chunk_plain as plain

TOP = {1: 448.0, 2: 127.0}  # DYNTS_CODE_E4M3, DYNTS_CODE_INT8


def hold(x, code):
    """bf16 [..., d] -> the values that the cache holds, in float64 (NaN for a block without a scale)."""
    y = x.double().unflatten(-1, (-1, 32))
    most = y.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(most) | (most >= 2.0 ** 126) | y.isnan().any(-1, keepdim=True)
    y, most = torch.where(bad, 0.0, y), torch.where(bad, 0.0, most)
    e = torch.full_like(most, -100.0)
    for k in range(-100, 127):  # the least that is enough, by trying
        e = torch.where((most > TOP[code] * 2.0 ** k), float(k + 1), e)
    unit = torch.tensor([2.0 ** k for k in range(-100, 128)], dtype=torch.float64)[(e + 100).long()]
    z = y / unit
    if code == 2:
        z = torch.round(z)
    else:
        step = torch.full_like(z, 2.0 ** -9)
        for k in range(-5, 9):
            step = torch.where(z.abs() >= 2.0 ** k, 2.0 ** (k - 3), step)
        z = torch.round(z / step) * step
    return torch.where(bad, math.nan, z * unit).flatten(-2)


def ancestors(parents, m):
    """[i][j]: token i sees token j, from a list of parents."""
    seen = torch.zeros((m, m), dtype=torch.bool)
    depth = []
    for i in range(m):
        p = parents[i]
        if 0 <= p < i:
            seen[i] = seen[p]
        seen[i, i] = True
        depth.append(depth[p] + 1 if 0 <= p < i else 0)
    return seen, depth


def words(seen, T):
    """[m][m] truth values as the words of T tokens: int32 [T][ceil(T / 32)]."""
    W = (T + 31) // 32
    out = torch.zeros((T, W), dtype=torch.int64)
    for i, j in seen.nonzero().tolist():
        out[i, j // 32] |= 1 << (j % 32)
    return torch.where(out >= 1 << 31, out - (1 << 32), out).to(torch.int32)


def attention(q, K, V, n, m, seen, scale):
    """One sequence's draft, the last m of n slots: q [T][Hq][d], K, V [Hkv][>= n][d], seen [m][m].  -> out, lse and their bounds, which are those of
    chunk_plain (the arithmetic is the same)."""
    Hq, d = q.shape[1:]
    Hkv = K.shape[0]
    half16, half32 = plain.HALF16, plain.HALF32
    q, K, V = q[:m].double(), K[:, :n].double(), V[:, :n].double()
    hidden = torch.zeros((m, n), dtype=torch.bool)
    hidden[:, n - m:] = ~seen
    r = dict(out=torch.zeros(m, Hq, d, dtype=torch.float64), lse=torch.zeros(m, Hq, dtype=torch.float64))
    r.update(out_tol=torch.zeros_like(r["out"]), lse_tol=torch.zeros_like(r["lse"]))
    for hq in range(Hq):
        h = hq // (Hq // Hkv)
        x = (q[:, hq] @ K[h].t()) * scale
        off = (d + 8) * half32 * (q[:, hq].abs() @ K[h].abs().t()) * scale + 8 * half32 * x.abs()
        x, off = x.masked_fill(hidden, -math.inf), off.masked_fill(hidden, 0.0)
        lse = torch.logsumexp(x, dim=-1)
        some = torch.isfinite(lse)
        at = torch.where(some, lse, 0.0)
        w = torch.where(~hidden & some[:, None], torch.exp(x - at[:, None]), 0.0)
        lse_tol = 1.5 * ((w * off).sum(-1) + (n + 8) * half32) + 8 * half32 * at.abs()
        rel = 1.5 * off + lse_tol[:, None] + 8 * half32 * (x.masked_fill(hidden, 0.0).abs() + at.abs()[:, None])
        spread = w @ V[h].abs()
        r["out"][:, hq], r["lse"][:, hq], r["lse_tol"][:, hq] = w @ V[h], lse, lse_tol
        r["out_tol"][:, hq] = half16 * (spread + r["out"][:, hq].abs()) * (1 + half16) + (w * 2 * rel) @ V[h].abs() + n * half32 * spread
    return r
