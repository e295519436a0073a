"""Chunks in the forms and with the inputs that tests/test_gpu_chunk.py does not bring together: positions far apart, the appending kernel in every
state of a cache, hidden keys in the kernels for many rows."""
import math

import pytest
import torch

from tests import chunk_plain as plain
from tests.test_gpu_chunk import Case

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def B():
    from paper_2601_18383_amd import binding
    return binding


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,d,Nb", [(8, 2, 64, 2), (28, 4, 128, 1), (32, 8, 128, 80), (16, 8, 64, 200)])
def test_a_bias_between_positions_far_apart(B, layout, Hq, Hkv, d, Nb):
    """A chunk's tokens up to 2^26 positions from its first one, a few from each other: whole distances as everywhere, exact below 2^24.  (By the distances
    from the chunk's first token, which have 24 bits, they were off by up to 4.)"""
    m = 5 if Nb < 80 else 72 * Hkv // Hq  # (72 rows of more than 512 units: the kernel for many rows)
    c = Case(B, layout, Hq, Hkv, d, [40] * Nb, [m] * Nb, seed=41)
    far = torch.cat((torch.tensor([100]), (1 << 26) + torch.cumsum(1 + torch.arange(m - 1) % 3, 0))).to(torch.int32)
    for b in range(Nb):
        c.pos[b][:, 40:] = far
    c.fill(True)
    slope = (0.5 * 2.0 ** (-4.0 * torch.arange(Hq) / Hq)).to(torch.float32)
    sh = B.Shaping(slope=slope.to(DEV))
    dst = torch.zeros((Nb, Hkv, c.cap), dtype=torch.float32, device=DEV)
    q = c.q.to(DEV)
    B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n, shaping=sh)
    B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n, shaping=sh)
    if Nb > 4:  # (the first and the last of them)
        for name in ("n_old", "n_new"):
            setattr(c, name, [getattr(c, name)[0], getattr(c, name)[-1]])
        for name in ("K", "V", "q", "pos", "out", "lse"):
            x = getattr(c, name)
            setattr(c, name, [x[0], x[-1]] if isinstance(x, list) else torch.stack((x[0], x[-1])))
        dst = torch.stack((dst[0], dst[-1]))
    c.check("far", lse=c.lse, recv=dst, slope=slope)
