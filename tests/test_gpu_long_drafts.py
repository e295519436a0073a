"""Attention of long drafts against the definition: more row blocks a unit than codes are converted for in the kernels themselves, many words a token."""
import pytest
import torch

from tests.test_gpu_tree import DEV, KINDS, Draft

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2601_18383_amd import binding
    return binding


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new,how", [
    (32, 8, 64, [50], [700], "any"),             # 22 blocks of 128 rows a unit
    (16, 4, 128, [50], [700], "deep"),
    (16, 4, 128, [33, 0], [1500, 3], "any"),     # 47 words
    (16, 16, 64, [100], [1300], "deep"),         # 11 blocks
    (8, 8, 128, [1], [1400], "chain"),           # 11 blocks: whole numbers are unpacked, e4m3 is not
])
def test_attend(B, kind, Hq, Hkv, d, n_old, n_new, how):
    Draft(B, kind, Hq, Hkv, d, n_old, n_new, how=how, seed=51).attend().check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_the_longest(B, kind, d):
    """4096 tokens, all of their rows, appended and attended in one call."""
    x = Draft(B, kind, 2, 1, d, [60], [4096], how="any", seed=52, append=False)
    taken = torch.zeros((1,), dtype=torch.int32, device=DEV)
    x.step(taken).check()
    assert taken.tolist() == [4096] and x.c.seq_len[0].tolist() == [4156] and int(x.c.status.item()) == 0
