"""Where the bias by distance is rounded in chunk_attend_few_kernel on bf16 caches, bit by bit: the first slot of a tile has the bias rounded and the logit's product
exact, the others the logit's product rounded and the bias exact.  Results of one build are those of the next."""
import math
from fractions import Fraction

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def B():
    from paper_2601_18383_amd import binding
    return binding


def _f32(x):
    """A Fraction rounded to fp32, ties to even (normal numbers)."""
    if x == 0:
        return Fraction(0)
    e = math.floor(math.log2(abs(x)))
    e = e if Fraction(2) ** e <= abs(x) else e - 1
    e = e if Fraction(2) ** (e + 1) > abs(x) else e + 1
    step = Fraction(2) ** (e - 23)
    return round(x / step) * step  # (Fraction's round is to even)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_a_row_that_sees_one_slot(B, d, paged):
    """The lse of a token that sees one slot is that slot's logit: 2^0 is the sum, and its logarithm 0."""
    gen = torch.Generator().manual_seed(d)
    Hq, n = 4, 70
    c = (B.PagedCache if paged else B.Cache)(1, 1, Hq, Hq, d, 80, 0, 0, 1)
    scratch = torch.empty(B.dynts_chunk_scratch_bytes(c.cfg, n), dtype=torch.uint8, device=DEV)
    k = torch.zeros((1, n, Hq, d), dtype=torch.bfloat16)
    q = torch.zeros((1, 8, Hq, d), dtype=torch.bfloat16)
    k[..., 3] = (1 + torch.rand((1, n, Hq), generator=gen)).to(torch.bfloat16)  # (one product a logit: exact)
    q[..., 3] = (1 + torch.rand((1, 8, Hq), generator=gen)).to(torch.bfloat16) * 4
    slope = torch.rand((Hq,), generator=gen) + 0.1
    B.dynts_chunk_append(c.ctx, 0, k.to(DEV), k.to(DEV), scratch)
    out, lse = torch.zeros((1, 8, Hq, d), dtype=torch.bfloat16, device=DEV), torch.zeros((1, 8, Hq), dtype=torch.float32, device=DEV)
    log2e, ln2 = Fraction(float(torch.tensor(1.4426950408889634))), Fraction(float(torch.tensor(0.6931471805599453)))
    scale = _f32(Fraction(float(torch.tensor(1.0) / torch.tensor(math.sqrt(d), dtype=torch.float32))) * log2e)
    differ = 0
    for first in range(0, n - 8, 8):  # token i sees slot first + i alone
        at = torch.arange(first, first + 8, dtype=torch.int32)[None]
        B.dynts_chunk_attend(c.ctx, 0, q.to(DEV), out, scratch, lse=lse, shaping=B.Shaping(slope=slope.to(DEV), first=at.to(DEV), last=at.to(DEV)))
        for i in range(8):
            for h in range(Hq):
                slot, own = first + i, n - 8 + i
                s, steep = Fraction(float(q[0, i, h, 3])) * Fraction(float(k[0, slot, h, 3])), _f32(Fraction(float(slope[h])) * log2e)
                whole = _f32(s * scale - _f32(steep * (own - slot))), _f32(_f32(s * scale) - steep * (own - slot))
                # (an element of the products is key 8 (e / 4) + 4 (lane / 32) + e % 4 of the tile: element 0 is slots 0 and 4)
                x = whole[0] if slot % 32 in (0, 4) else whole[1]
                differ += whole[0] != whole[1]
                assert float(lse[0, i, h]) == float(_f32(x * ln2)), (slot, h)
    assert differ > 40
