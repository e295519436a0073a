"""dynts_tree_keep while a score update is owed: tokens drafted by single steps, of which a path is kept."""
import pytest
import torch

from tests.test_gpu_tree import DEV, _cache, _ints, _rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2601_18383_amd import binding
    return binding


@pytest.mark.parametrize("then", ["update", "step"])
@pytest.mark.parametrize("owed", ["step", "hinted step", "attention", "kept logits", "step before the draft"])
@pytest.mark.parametrize("kind", ["dense", "paged"])
def test_an_owed_update_is_of_the_rows_as_they_lay(B, kind, owed, then):
    """Scores, rows and lengths are those of a cache whose update was asked for before the path was kept."""
    gen = torch.Generator().manual_seed(41)
    Nb, Hq, Hkv, d, T = 3, 8, 2, 128, 9
    caches = [_cache(B, kind, Nb, Hq, Hkv, d, 200) for _ in range(2)]
    K0, V0, m0 = _rand(gen, Nb, Hkv, 70, d).to(DEV), _rand(gen, Nb, Hkv, 70, d).to(DEV), _ints([59, 70, 3])
    steps = [(_rand(gen, Nb, Hq, d, scale=1.5).to(DEV), _rand(gen, Nb, Hkv, d).to(DEV), _rand(gen, Nb, Hkv, d).to(DEV)) for _ in range(5 + T)]
    parents = _ints([[-1, 0, 0, 1, 2, 3, 4, 5, 6], [-1, -1, 0, 1, 2, 3, 4, 4, 4], [i - 1 for i in range(T)]])
    leaf, paths = _ints([8, 7, 3]), [[0, 2, 4, 6, 8], [0, 2, 4, 7], [0, 1, 2, 3]]
    before = [1 if owed == "step before the draft" else 0]
    for c, asks in zip(caches, (False, True)):
        out = torch.zeros((Nb, Hq, d), dtype=torch.float32, device=DEV)
        B.dynts_prefill(c.ctx, 0, K0, V0, m0)
        drafted = steps[:5] if before[0] else steps
        for i, (q, k, v) in enumerate(drafted):
            if owed in ("attention", "kept logits"):
                B.dynts_append(c.ctx, 0, k, v)
                B.dynts_decode_attend(c.ctx, 0, q, out)
                if owed == "kept logits" and i < len(steps) - 1:  # (left where the update has been seen to follow)
                    B.dynts_update_scores(c.ctx, 0)
            else:
                if owed == "hinted step" and i == len(steps) - 1:
                    B.dynts_hint_trigger(c.ctx, 0)
                B.dynts_decode_step(c.ctx, 0, q, k, v, out)
        if before[0]:
            rows = lambda at: torch.stack([s[at] for s in steps[5:]], dim=1).contiguous()
            scratch = torch.empty(B.dynts_chunk_scratch_bytes(c.cfg, T), dtype=torch.uint8, device=DEV)
            B.dynts_chunk_append(c.ctx, 0, rows(1), rows(2), scratch)
        seen, kept = torch.zeros((Nb, T, 1), dtype=torch.int32, device=DEV), torch.zeros((Nb,), dtype=torch.int32, device=DEV)
        B.dynts_tree_build(parents, seen)
        if asks:
            B.dynts_update_scores(c.ctx, 0)
        B.dynts_tree_keep(c.ctx, 0, seen, leaf, None, kept)
        assert kept.tolist() == [5, 4, 4]
        if then == "update":
            B.dynts_update_scores(c.ctx, 0)
        for _ in range(2):  # (the first of which would apply it otherwise, to the row that it appends as well)
            B.dynts_decode_step(c.ctx, 0, *steps[0], out)
        B.dynts_update_scores(c.ctx, 0)
    a, b = caches
    n = a.seq_len[0].tolist()
    assert n == [59 + 5 + 5 + 2, 70 + 5 + 4 + 2, 3 + 5 + 4 + 2] and torch.equal(a.seq_len, b.seq_len) and torch.equal(a.next_pos, b.next_pos)
    Ka, Kb = a.K[0], b.K[0]
    for i in range(Nb):
        assert torch.equal(a.S[0, i, :, :n[i]], b.S[0, i, :, :n[i]]) and torch.equal(a.pos[0, i, :, :n[i]], b.pos[0, i, :, :n[i]])
        assert torch.equal(Ka[i, :, :n[i]], Kb[i, :, :n[i]])
        rows = torch.stack([steps[5 + t][1][i] for t in paths[i]], dim=1)  # [Hkv][kept][d]
        assert torch.equal(Ka[i, :, n[i] - 2 - len(paths[i]):n[i] - 2], rows)
    if kind == "paged":
        assert all(len(set(c.pages_in_use())) == 1 for c in caches)
