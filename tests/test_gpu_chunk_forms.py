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


# ---- the kernel that appends a chunk's rows itself, in every state of a cache ---------------------------------------------

LONG = [  # Hq, Hkv, d, n_old, n_new: sizes that go to chunk_attend_kernel
    (32, 8, 128, [0, 1, 31, 32, 33, 64, 100, 200, 5], [40, 33, 40, 1, 0, 40, 39, 40, 17]),
    (16, 8, 64, [0, 7, 64, 130] * 5, [50, 49, 1, 32] * 5),
    (28, 4, 128, [90, 0, 257] * 5, [64, 60, 31] * 5),
    (8, 2, 128, [8000], [600]),                              # its keys in shares
]


def few_rows(c):
    """Whether the chunks of a case go to chunk_attend_few_kernel: the line that chunk.hip draws."""
    R, units = c.T * (c.Hq // c.Hkv), len(c.n_old) * c.Hkv
    F = units * ((R + 31) // 32)
    return R <= 32 or (F <= (256 if c.d == 128 else 512) and (R <= 64 or F * c.cap <= 1 << 20))


def state_of(cache, b, rows):
    """What sequence b has in the cache, its first `rows` slots (those behind its length belong to no page)."""
    c = cache
    return [x.clone() for x in (c.K[0, b, :, :rows], c.V[0, b, :, :rows], c.S[0, b], c.pos[0, b], c.seq_len[0, b], c.next_pos[0, b], c.n_prompt[b])]


def check_rows(c, b, n):
    K, V = c.cache.K[0, b, :, :n].cpu(), c.cache.V[0, b, :, :n].cpu()
    assert torch.equal(K, c.K[b, :, :n]) and torch.equal(V, c.V[b, :, :n])
    assert torch.equal(c.cache.pos[0, b, :, :n].cpu(), c.pos[b][:, :n])


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", LONG)
def test_a_question_in_long_chunks(B, layout, Hq, Hkv, d, n_old, n_new):
    """Slots of infinite score, n_prompt moves on; of two sequences that have thinking tokens the one with a question is refused, and nothing of it is touched."""
    c = Case(B, layout, Hq, Hkv, d, n_old, n_new, gaps=7, seed=51)
    assert not few_rows(c)
    c.fill(False)
    c.cache.n_prompt.copy_(torch.tensor(n_old, dtype=torch.int32))
    thinking = [b for b, a in enumerate(n_old) if a][:2] if len(n_old) > 1 else []
    for b, a in enumerate(n_old):
        c.cache.S[0, b, :, :a] = math.inf
    for b in thinking:
        c.cache.n_prompt[b] = n_old[b] - 1
        c.cache.S[0, b, :, n_old[b] - 1] = 0.25
    refused = [b for b in thinking if n_new[b]]
    before = {b: state_of(c.cache, b, n_old[b]) for b in refused}
    B.dynts_chunk_step(c.cache.ctx, 0, c.q.to(DEV), c.k_new, c.v_new, c.out, c.scratch, lse=c.lse, n_new=c.n, question=True)
    assert int(c.cache.status.item()) == (8 if refused else 0)
    for b in refused:
        assert torch.all(c.out[b] == 7.0) and torch.all(c.lse[b] == 7.0)
        assert all(torch.equal(x, y) for x, y in zip(before[b], state_of(c.cache, b, n_old[b])))
        c.n_new = c.n_new[:b] + [0] + c.n_new[b + 1:]
    c.check("question", lse=c.lse)
    for b, (a, m) in enumerate(zip(n_old, c.n_new)):
        n = a + m
        check_rows(c, b, n)
        assert [int(x[0, b]) for x in (c.cache.seq_len, c.cache.next_pos)] == [n, c.next[b] + m]
        assert torch.all(c.cache.S[0, b, :, n:] == 0)
        if b not in thinking:
            assert int(c.cache.n_prompt[b]) == n and torch.all(c.cache.S[0, b, :, :n] == math.inf)


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", LONG)
def test_scores_from_outside_in_long_chunks(B, layout, Hq, Hkv, d, n_old, n_new):
    c = Case(B, layout, Hq, Hkv, d, n_old, n_new, external=True, seed=52)
    assert not few_rows(c)
    c.fill(False)
    c.cache.S.fill_(0.5)
    s = torch.rand((len(n_old), c.T, Hkv), generator=c.gen).to(DEV)
    B.dynts_chunk_step(c.cache.ctx, 0, c.q.to(DEV), c.k_new, c.v_new, c.out, c.scratch, n_new=c.n, s_new=s)
    c.check("external")
    for b, (a, m) in enumerate(zip(n_old, n_new)):
        check_rows(c, b, a + m)
        want = torch.full_like(c.cache.S[0, b], 0.5)
        want[:, a:a + m] = s[b, :m].t()
        assert torch.equal(c.cache.S[0, b], want)
    assert int(c.cache.status.item()) == 0


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", LONG[:3])
def test_long_chunks_that_do_not_fit(B, layout, Hq, Hkv, d, n_old, n_new):
    """One slot too few for the sequence that would be longest: it is left alone, the others are not."""
    longest = max(a + m for a, m in zip(n_old, n_new))
    c = Case(B, layout, Hq, Hkv, d, n_old, n_new, seed=53, spare=0)
    c.cache.close()
    c.cap = longest - 1
    c.cache = (B.Cache if layout == "dense" else B.PagedCache)(1, len(n_old), Hq, Hkv, d, c.cap, 0, 0, 1)
    c.K, c.V = c.K[:, :, :c.cap], c.V[:, :, :c.cap]
    assert not few_rows(c)
    over = [b for b, (a, m) in enumerate(zip(n_old, n_new)) if a + m == longest]
    c.fill(False)
    before = {b: state_of(c.cache, b, n_old[b]) for b in over}
    B.dynts_chunk_step(c.cache.ctx, 0, c.q.to(DEV), c.k_new, c.v_new, c.out, c.scratch, lse=c.lse, n_new=c.n)
    assert int(c.cache.status.item()) == 1
    for b in over:
        assert torch.all(c.out[b] == 7.0) and torch.all(c.lse[b] == 7.0)
        assert all(torch.equal(x, y) for x, y in zip(before[b], state_of(c.cache, b, n_old[b])))
        c.n_new = c.n_new[:b] + [0] + c.n_new[b + 1:]
    c.check("fits", lse=c.lse)
    for b, (a, m) in enumerate(zip(n_old, c.n_new)):
        check_rows(c, b, a + m)
    if layout == "paged":
        used, taken = c.cache.pages_in_use()
        assert used == taken


def test_long_chunks_on_a_pool_without_enough_pages(B):
    """Whichever sequences get pages have their whole chunk, the others keep what they had; no page is lost."""
    c = Case(B, "paged", 32, 8, 128, [64] * 9, [70] * 9, seed=54)
    assert not few_rows(c)
    c.cache.close()
    c.cache = B.PagedCache(1, 9, 32, 8, 128, c.cap, 0, 0, 1, n_pages=9 * 8 + 4 * 16 + 5)  # two more pages a head: four chunks' worth
    c.fill(False)
    before = [state_of(c.cache, b, 64) for b in range(9)]
    B.dynts_chunk_step(c.cache.ctx, 0, c.q.to(DEV), c.k_new, c.v_new, c.out, c.scratch, lse=c.lse, n_new=c.n)
    assert int(c.cache.status.item()) == 4 and int(c.cache.free_top.item()) == 5
    lens = c.cache.seq_len[0].tolist()
    assert sorted(lens) == [64] * 5 + [134] * 4
    for b in range(9):
        if lens[b] == 64:
            assert torch.all(c.out[b] == 7.0) and torch.all(c.lse[b] == 7.0)
            assert all(torch.equal(x, y) for x, y in zip(before[b], state_of(c.cache, b, 64)))
            c.n_new = c.n_new[:b] + [0] + c.n_new[b + 1:]
        else:
            check_rows(c, b, 134)
    c.check("pages", lse=c.lse)
    used, taken = c.cache.pages_in_use()
    assert used == taken


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,d,Nb,T", [(32, 8, 128, 9, 40), (16, 8, 64, 20, 50), (8, 2, 128, 1, 600)])
def test_captured_long_steps(B, layout, Hq, Hkv, d, Nb, T):
    """A long chunk's step recorded once and replayed, each time on a longer cache, with eager work in between: the same as eager steps."""
    start = 7000 if Nb == 1 else 10
    c, e = (Case(B, layout, Hq, Hkv, d, [start] * Nb, [T] * Nb, seed=55, spare=4 * T).fill(False) for _ in range(2))
    assert not few_rows(c)
    q = c.q.to(DEV)
    run = lambda x: B.dynts_chunk_step(x.cache.ctx, 0, q, x.k_new, x.v_new, x.out, x.scratch, lse=x.lse)
    B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch)  # (what the library loads with its first launch is not recorded)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(c)
    assert int(c.cache.seq_len[0, 0]) == start
    for turn in range(4):
        graph.replay()
        run(e)
        torch.cuda.synchronize()
        n = start + (turn + 1) * T
        assert c.cache.seq_len[0].tolist() == [n] * Nb
        for name in ("out", "lse"):
            assert torch.equal(getattr(c, name), getattr(e, name)), (name, turn)
        for name in ("K", "V", "pos", "S"):
            assert torch.equal(getattr(c.cache, name)[..., :n, :] if name in "KV" else getattr(c.cache, name)[..., :n],
                               getattr(e.cache, name)[..., :n, :] if name in "KV" else getattr(e.cache, name)[..., :n]), (name, turn)
        c.scratch.fill_(turn)
        c.out.fill_(7.0)
    assert int(c.cache.status.item()) == 0


def test_long_steps_on_two_streams_at_once(B):
    """Two caches, each with a scratch and a stream of its own: what each gives alone."""
    cases = [Case(B, layout, *shape, seed=56).fill(False) for layout, shape in (("dense", LONG[0]), ("paged", LONG[3]))]
    qs = [c.q.to(DEV) for c in cases]

    def back(c):
        c.cache.seq_len[0].copy_(torch.tensor(c.n_old, dtype=torch.int32))
        c.cache.next_pos[0].copy_(torch.tensor(c.next, dtype=torch.int32))
        c.cache.S.zero_()
        c.out.fill_(7.0)

    step = lambda c, q: B.dynts_chunk_step(c.cache.ctx, 0, q, c.k_new, c.v_new, c.out, c.scratch, lse=c.lse, n_new=c.n)
    attend = lambda c, q: B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n)
    want = []
    dense = cases[:1]  # (a paged sequence set back by its length alone would keep its pages: its chunk, once in, is attended again)
    for c, q in zip(cases, qs):
        step(c, q)
        c.check("alone", lse=c.lse)
        if c not in dense:
            attend(c, q)
            c.check("alone", lse=c.lse)
        want.append([x.clone() for x in (c.out, c.lse, c.cache.S)])
    streams = [torch.cuda.Stream() for _ in cases]
    for turn in range(4):
        for c in dense:
            back(c)
        torch.cuda.synchronize()
        for c, q, stream in zip(cases, qs, streams):
            with torch.cuda.stream(stream):
                (step if c in dense else attend)(c, q)
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert torch.equal(c.lse, w[1]) and torch.equal(c.out, w[0])
        for c, w in zip(dense, want):
            assert torch.equal(c.cache.S, w[2])


# ---- what else the kernels for many rows have not met -------------------------------------------------------------------

@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,d,Nb,T", [(32, 8, 128, 9, 70), (16, 8, 64, 20, 70), (28, 4, 128, 20, 64)])
@pytest.mark.parametrize("biased", [False, True])
def test_keys_hidden_from_all_may_be_anything_for_many_rows(B, layout, Hq, Hkv, d, Nb, T, biased):
    """K rows of another document that hold NaN and infinities, some of them in a tile with rows that are seen."""
    c = Case(B, layout, Hq, Hkv, d, [100] * Nb, [T] * Nb, seed=57)
    assert not few_rows(c)
    real = c.K.clone()
    c.K[:, :, :40] = math.nan
    c.K[:, :, 40:50] = math.inf
    c.fill(True)
    c.K = real
    first = torch.full((Nb, T), 50, dtype=torch.int32)
    slope = (2.0 ** (-8.0 * (1 + torch.arange(Hq)) / Hq)).to(torch.float32) if biased else None
    shape = dict(first=first, **({"slope": slope} if biased else {}))
    sh = B.Shaping(**{k: v.to(DEV) for k, v in shape.items()})
    q = c.q.to(DEV)
    dst = torch.zeros((Nb, Hkv, c.cap), dtype=torch.float32, device=DEV)
    B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n, shaping=sh)
    B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n, shaping=sh)
    assert torch.all(dst[:, :, :50] == 0)
    c.check("hidden", lse=c.lse, recv=dst, **shape)


@pytest.mark.parametrize("shape", [dict(), dict(softcap=4.0), dict(softcap=4.0, window=30)])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", LONG[:2])
def test_a_scale_of_the_callers_for_many_rows(B, shape, Hq, Hkv, d, n_old, n_new):
    c = Case(B, "dense", Hq, Hkv, d, n_old, n_new, seed=58)
    assert not few_rows(c)
    c.cache.close()
    c.cache = B.Cache(1, len(n_old), Hq, Hkv, d, c.cap, 0, 0, 1, softmax_scale=0.31)
    c.fill(True)
    q = c.q.to(DEV)
    sh = B.Shaping(**shape) if shape else None
    dst = torch.zeros((len(n_old), Hkv, c.cap), dtype=torch.float32, device=DEV)
    B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n, shaping=sh)
    B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n, shaping=sh)
    c.check("scale", lse=c.lse, recv=dst, scale=0.31, **shape)


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", LONG)
def test_many_rows_do_not_change_from_run_to_run(B, layout, Hq, Hkv, d, n_old, n_new):
    c = Case(B, layout, Hq, Hkv, d, n_old, n_new, gaps=9, seed=59).fill(True)
    assert not few_rows(c)
    q = c.q.to(DEV)
    for sh in (None, B.Shaping(softcap=20.0, window=60), B.Shaping(slope=torch.full((Hq,), 0.1, device=DEV))):
        first = None
        for turn in range(4):
            c.scratch.fill_(turn)
            B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n, shaping=sh)
            dst = torch.zeros((len(n_old), Hkv, c.cap), dtype=torch.float32, device=DEV)
            B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n, shaping=sh)
            got = (c.out.clone(), c.lse.clone(), dst)
            first = first or got
            assert all(torch.equal(x, y) for x, y in zip(first, got))


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,d,Nb,T", [(28, 4, 128, 3, 6), (8, 2, 64, 5, 9), (32, 8, 128, 9, 40)])
def test_drafts_that_are_taken_back(B, layout, Hq, Hkv, d, Nb, T):
    """Drafted tokens are appended and attended, some are dropped again, and only those that stay give weights to the slots: the cache of one that never
    saw the others."""
    n_old, kept = [70 + 3 * b for b in range(Nb)], [(T * (b + 1)) // Nb for b in range(Nb)]  # (the last sequence keeps all)
    a = Case(B, layout, Hq, Hkv, d, n_old, [T] * Nb, gaps=5, seed=60).fill(False)
    b = Case(B, layout, Hq, Hkv, d, n_old, [T] * Nb, gaps=5, seed=60).fill(False)
    q = a.q.to(DEV)
    stay = torch.tensor(kept, dtype=torch.int32, device=DEV)
    B.dynts_chunk_append(a.cache.ctx, 0, a.k_new, a.v_new, a.scratch)
    B.dynts_chunk_attend(a.cache.ctx, 0, q, a.out, a.scratch, lse=a.lse)
    c = a.cache
    c.keep_idx.copy_(torch.arange(a.cap, device=DEV, dtype=torch.int32).expand_as(c.keep_idx))
    B.dynts_compact(c.ctx, 0, c.keep_idx, (c.seq_len[0] - T + stay).to(torch.int32))
    c.next_pos[0] -= T - stay
    B.dynts_chunk_scores(c.ctx, 0, q, a.lse, n_new=stay)
    B.dynts_chunk_step(b.cache.ctx, 0, q, b.k_new, b.v_new, b.out, b.scratch, lse=b.lse, n_new=stay)
    assert torch.equal(a.cache.seq_len, b.cache.seq_len) and torch.equal(a.cache.next_pos, b.cache.next_pos)
    for i, (n, m) in enumerate(zip(n_old, kept)):
        for x, y in zip(state_of(a.cache, i, n + m)[:2], state_of(b.cache, i, n + m)[:2]):
            assert torch.equal(x, y)
        assert torch.equal(a.cache.pos[0, i, :, :n + m], b.cache.pos[0, i, :, :n + m])
        # (lse and weights of either are off by roundings of the definition's)
        r = plain.attention(a.q[i], a.K[i], a.V[i], a.pos[i], n + m, m, 1.0 / math.sqrt(d)) if m else None
        for x in (a, b):
            if m:
                plain.check(x.out[i, :m], r["out"], r["out_tol"], "out")
                plain.check(x.cache.S[0, i, :, :n + m], r["recv"], r["recv_tol"], "S")
    if layout == "paged":
        used, taken = a.cache.pages_in_use()
        assert used == taken
    assert int(a.cache.status.item()) == 0 and int(b.cache.status.item()) == 0
