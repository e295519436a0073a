"""Caps on a chunk's logits that lie far above them, and the least ones: a logit keeps its own bits under any cap."""
import ctypes as C
import math

import pytest
import torch

from tests import chunk_plain as plain
from tests.chunk_plain import HALF16, HALF32
from tests.test_gpu_chunk import Case

DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def B():
    from paper_2601_18383_amd import binding, build
    if build.is_stale():
        build.build()
    return binding


def test_caps_below_the_smallest_normal_numbers_are_refused(B):
    """2 log2 e * scale / softcap has to be finite: with it infinite a logit of 0 would be capped to NaN.  Every other cap is taken (the null output
    is what these calls are refused for)."""
    one = C.c_void_p(256)
    cfg = B.make_config(1, 3, 8, 2, 128, 400, 0, 0, 1)
    ctx = B.dynts_create(cfg)
    assert B.lib.dynts_bind(ctx, *([one] * 7), one, B.dynts_workspace_bytes(cfg), one) == B.DYNTS_OK
    need = B.dynts_chunk_scratch_bytes(cfg, 16)

    def calls(softcap):
        sh = C.byref(B.dynts_shaping(softcap, 0, None, None, None))
        return (B.lib.dynts_chunk_attend(ctx, 0, one, 16, None, sh, None, None, one, need, None),
                B.lib.dynts_chunk_scores(ctx, 0, one, 16, None, sh, None, None, 1, None),
                B.lib.dynts_chunk_step(ctx, 0, one, one, one, None, 16, None, 0, sh, None, None, one, need, None))

    for softcap in (1e-45, 1e-40, 7e-40):
        assert calls(softcap) == (B.DYNTS_EINVAL,) * 3, softcap
    for softcap in (1e-37, 1e-3, 1.0, 50.0, 1e6, 1.2e38, 3.4e38):
        assert calls(softcap) == (B.DYNTS_ENULL,) * 3, softcap
    B.dynts_destroy(ctx)


def capped(c, b, softcap, slope, logit_off):
    """Sequence b of a case in float64, as chunk_plain.attention has it, where the cap's share of a logit's error is logit_off(x)."""
    a, m, d, G = c.n_old[b], c.n_new[b], c.d, c.Hq // c.Hkv
    n = a + m
    q, K, V = (x.double() for x in (c.q[b, :m], c.K[b, :, :n], c.V[b, :, :n]))
    pos = c.pos[b][:, :n].long()
    r = {k: torch.zeros(s, dtype=torch.float64) for k, s in (("out", (m, c.Hq, d)), ("out_tol", (m, c.Hq, d)), ("lse", (m, c.Hq)), ("lse_tol", (m, c.Hq)),
                                                           ("recv", (c.Hkv, n)), ("recv_tol", (c.Hkv, n)))}
    for hq in range(c.Hq):
        h = hq // G
        x = (q[:, hq] @ K[h].t()) / math.sqrt(d)
        off = (d + 8) * HALF32 * (q[:, hq].abs() @ K[h].abs().t()) / math.sqrt(d) + 8 * HALF32 * x.abs()
        x = softcap * torch.tanh(x / softcap)
        off = off + logit_off(x)
        if slope is not None:
            bias = float(slope[hq]) * (pos[h, a:n, None] - pos[h][None]).abs().double()
            x, off = x - bias, off + 8 * HALF32 * bias
        x = torch.where(torch.arange(n)[None] <= a + torch.arange(m)[:, None], x, -math.inf)
        off = torch.where(torch.isfinite(x), off, 0.0)
        lse = torch.logsumexp(x, dim=-1)
        w = torch.exp(x - lse[:, None])
        # (the bounds of chunk_plain.attention)
        lse_tol = 1.5 * ((w * off).sum(-1) + (n + 8) * HALF32) + 8 * HALF32 * lse.abs()
        rel = 1.5 * off + lse_tol[:, None] + 8 * HALF32 * (torch.where(torch.isfinite(x), x, 0.0).abs() + lse.abs()[:, None])
        spread = w @ V[h].abs()
        r["out"][:, hq] = w @ V[h]
        r["out_tol"][:, hq] = HALF16 * (spread + r["out"][:, hq].abs()) * (1 + HALF16) + (w * 2 * rel) @ V[h].abs() + n * HALF32 * spread
        r["lse"][:, hq], r["lse_tol"][:, hq] = lse, lse_tol
        r["recv"][h] += w.sum(0)
        r["recv_tol"][h] += (w * (torch.exp(rel) - 1)).sum(0) + (m * G + 8) * HALF32 * w.sum(0) + m * 2.0 ** -126
    return r


@pytest.mark.gpu
@pytest.mark.parametrize("softcap", [0.01, 127.0, 128.0, 129.0, 700.0, 1e5, 1e9, 1e30, 1.2e38, 3.4e38])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", [
    (28, 4, 128, [0, 70], [37, 4]),                              # few rows
    (8, 2, 64, [300, 1, 64], [1, 1, 1]),                         # single tokens
    (32, 8, 128, [0, 200, 33] * 3, [64, 40, 50] * 3),            # 288 workgroups of 32 rows and more: many rows
    (16, 8, 64, [0, 1, 63, 200] * 4, [150, 149, 64, 1] * 4),     # many rows
])
def test_a_cap_leaves_a_logit_its_bits(B, softcap, biased, Hq, Hkv, d, n_old, n_new):
    """Up to 128 off by 6 half steps of the cap at most (the bound of 8 that chunk_plain has); above, by 24 of the capped logit: whichever form a logit takes there,
    |z| < 0.3 or not, see soft_cap_far.  Logits of up to several hundred: on both sides of 0.3 of the middle caps."""
    c = Case(B, "dense", Hq, Hkv, d, n_old, n_new, gaps=30, seed=31, qscale=60.0 if softcap < 1e4 else 3.0).fill(True)
    slope = (2.0 ** (-8.0 * (1 + torch.arange(Hq)) / Hq)).to(torch.float32) if biased else None
    sh = B.Shaping(softcap=softcap, slope=slope.to(DEV) if biased else None)
    softcap = float(torch.tensor(softcap, dtype=torch.float32))
    dst = torch.full((len(n_old), Hkv, c.cap), 7.0, dtype=torch.float32, device=DEV)
    q = c.q.to(DEV)
    B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n, shaping=sh)
    B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n, shaping=sh)
    off = (lambda x: 24 * HALF32 * x.abs()) if softcap > 128 else (lambda x: 8 * HALF32 * softcap)
    for b, (a, m) in enumerate(zip(n_old, n_new)):
        r = capped(c, b, softcap, slope, off)
        plain.check(c.out[b, :m], r["out"], r["out_tol"], "out[%d]" % b)
        plain.check(c.lse[b, :m], r["lse"], r["lse_tol"], "lse[%d]" % b)
        plain.check(dst[b, :, :a + m], r["recv"], r["recv_tol"], "received[%d]" % b)
