"""Drafts that branch (dynts_tree_*) against the definition in float64 and against chunks."""
import math

import pytest
import torch

from tests import chunk_plain as plain
from tests import codes_plain as held

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
KINDS = ["dense", "paged", "e4m3", "int8", "e4m3_paged", "int8_paged"]


@pytest.fixture(scope="module")
def B():
    from paper_2601_18383_amd import binding
    return binding


def _rand(gen, *shape, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(torch.bfloat16)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _parents(gen, T, how):
    if how == "chain":
        return [i - 1 for i in range(T)]
    if how == "flat":
        return [-1] * T
    if how == "deep":
        return [max(-1, i - 1 - int(torch.randint(0, 3, (1,), generator=gen))) for i in range(T)]
    return [int(torch.randint(-1, i, (1,), generator=gen)) if i else -1 for i in range(T)]


def _code(kind):
    return 1 if "e4m3" in kind else 2 if "int8" in kind else 0


def _cache(B, kind, Nb, Hq, Hkv, d, cap, L=1, external=False, **kw):
    if _code(kind):
        return B.CodedCache(L, Nb, Hq, Hkv, d, cap, 0, 0, 1, code=_code(kind), paged="paged" in kind, external_scores=external, **kw)
    return (B.PagedCache if kind == "paged" else B.Cache)(L, Nb, Hq, Hkv, d, cap, 0, 0, 1, external_scores=external, **kw)


def _values(x, kind):
    return held.hold(x, _code(kind)) if _code(kind) else x.double()


# ---- who sees whom -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("how", ["chain", "flat", "deep", "any"])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 64, 100, 257, 700])
def test_build(B, T, how):
    gen = torch.Generator().manual_seed(T)
    n_new = [T, T // 2, 0, max(1, T - 1), 2 * T, -4]
    parents = [_parents(gen, T, how) for _ in n_new]
    for b in (1, 3):  # padding holds anything
        for i in range(n_new[b], T):
            parents[b][i] = 12345 * (i + 1) if i % 2 else -(1 << 31)
    W = (T + 31) // 32
    seen, depth = torch.full((6, T, W), 77, dtype=torch.int32, device=DEV), torch.full((6, T), 77, dtype=torch.int32, device=DEV)
    B.dynts_tree_build(_ints(parents), seen, depth=depth, n_new=_ints(n_new))
    for b, m in enumerate(n_new):
        m = max(0, min(m, T))
        ref, deep = held.ancestors(parents[b], m)
        assert torch.equal(seen[b].cpu(), held.words(ref, T)), (b, m)
        assert depth[b].tolist() == deep + [0] * (T - m)
    again = torch.zeros_like(seen)
    B.dynts_tree_build(_ints(parents), again, n_new=_ints(n_new))  # without depths
    assert torch.equal(again, seen)


def test_build_of_parents_that_are_none(B):
    """A parent that is not before its child counts as the cache: no cycle, no token behind."""
    parents = [[5, 1, -7, 3, 3, 4, 1 << 30, -(1 << 31), 6, 9]]
    seen, depth = torch.zeros((1, 10, 1), dtype=torch.int32, device=DEV), torch.zeros((1, 10), dtype=torch.int32, device=DEV)
    B.dynts_tree_build(_ints(parents), seen, depth=depth)
    ref, deep = held.ancestors(parents[0], 10)
    assert torch.equal(seen[0].cpu(), held.words(ref, 10)) and depth[0].tolist() == deep
    long = [[i - 1 for i in range(4096)]]
    seen, depth = torch.zeros((1, 4096, 128), dtype=torch.int32, device=DEV), torch.zeros((1, 4096), dtype=torch.int32, device=DEV)
    B.dynts_tree_build(_ints(long), seen, depth=depth)
    assert depth[0].tolist() == list(range(4096)) and torch.all(seen[0, 4095] == -1) and int((seen[0, 2047] != 0).sum()) == 64


# ---- attention -----------------------------------------------------------------------------------------------------------

SHAPES = [  # Hq, Hkv, d, n_old, n_new
    (8, 2, 64, [0, 1, 63, 64, 200, 129, 31], [1, 1, 2, 3, 1, 5, 0]),
    (28, 4, 128, [0, 5, 300, 64, 31], [37, 0, 12, 40, 33]),             # odd groups, an empty draft, an empty cache
    (6, 6, 128, [130, 77], [33, 65]),                                   # no sharing of KV heads
    (16, 1, 64, [500, 3], [9, 100]),                                    # the largest group
    (16, 1, 128, [40], [257]),
    (8, 1, 128, [3000, 10], [20, 4]),                                   # keys in shares; a short cache beside it
    (8, 1, 64, [4000, 900], [64, 1]),
    (28, 4, 128, [0, 31, 32, 33, 100, 257, 64, 1, 5, 0, 90, 128], [60, 60, 1, 59, 0, 33, 60, 37, 32, 31, 64, 7]),  # many rows of many units
    (16, 8, 64, [0, 1, 63, 64, 65, 200, 31, 0] * 2, [150, 149, 64, 1, 0, 128, 65, 150] * 2),
    (8, 2, 128, [8000], [600]),                                         # many rows of few units: keys in shares
]


class Draft:
    """Caches of n_old slots and drafts of n_new tokens (appended, unless by the call under test)."""

    def __init__(self, B, kind, Hq, Hkv, d, n_old, n_new, how="any", seed=0, append=True, T=None, spare=5, external=False, masks=None, L=1, short=0, **kw):
        gen = self.gen = torch.Generator().manual_seed(seed + d + Hq)
        self.B, self.kind, self.Hq, self.Hkv, self.d, self.n_old, self.n_new = B, kind, Hq, Hkv, d, n_old, n_new
        Nb, self.T = len(n_old), T or max(max(n_new), 1)
        T = self.T
        self.cap = max(a + m for a, m in zip(n_old, n_new)) + spare
        self.c = c = _cache(B, kind, Nb, Hq, Hkv, d, self.cap - short, L=L, external=external, **kw)
        K, V = _rand(gen, Nb, self.cap, Hkv, d), _rand(gen, Nb, self.cap, Hkv, d)
        self.q = _rand(gen, Nb, T, Hq, d, scale=1.5)
        self.s = torch.rand((Nb, self.cap, Hkv), generator=gen)
        self.external = external
        self.scratch = torch.empty(B.dynts_codes_scratch_bytes(c.cfg, max(T, self.cap)), dtype=torch.uint8, device=DEV)
        self.scratch.fill_(0xA5)
        total = [a + (m if append else 0) for a, m in zip(n_old, n_new)]
        for layer in range(L):
            B.dynts_chunk_append(c.ctx, layer, K.to(DEV), V.to(DEV), self.scratch, n_new=_ints(total), s_new=self.s.to(DEV) if external else None)
        pad = lambda x, fill: torch.stack([torch.cat((x[b, a:a + m], torch.full((T - m, *x.shape[2:]), fill, dtype=x.dtype)))
                                           for b, (a, m) in enumerate(zip(n_old, n_new))]).contiguous().to(DEV)
        self.k_new, self.v_new, self.s_new = pad(K, math.nan), pad(V, math.nan), pad(self.s, math.nan)
        for b, m in enumerate(n_new):
            self.q[b, m:] = math.nan
        self.K, self.V = _values(K, kind).transpose(1, 2), _values(V, kind).transpose(1, 2)
        self.parents = [_parents(gen, T, how) for _ in n_old]
        if masks:
            self.masks = [masks(gen, m) for m in n_new]
            self.seen = torch.stack([held.words(x, T) for x in self.masks]).to(DEV)
        else:
            self.masks = [held.ancestors(p, m)[0] for p, m in zip(self.parents, n_new)]
            self.seen = torch.zeros((Nb, T, (T + 31) // 32), dtype=torch.int32, device=DEV)
            B.dynts_tree_build(_ints(self.parents), self.seen, n_new=_ints(n_new))
        self.out = torch.full((Nb, T, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((Nb, T, Hq), 7.0, dtype=torch.float32, device=DEV)
        self.n = _ints(n_new)

    def attend(self, layer=0):
        self.B.dynts_tree_attend(self.c.ctx, layer, self.q.to(DEV), self.seen, self.out, self.scratch, lse=self.lse, n_new=self.n)
        return self

    def step(self, taken, layer=0):
        self.B.dynts_tree_step(self.c.ctx, layer, self.q.to(DEV), self.k_new, self.v_new, self.seen, taken, self.out, self.scratch, lse=self.lse,
                               n_new=self.n, s_new=self.s_new if self.external else None)
        return self

    def check(self, skip=()):
        worst = {}
        for b, (a, m) in enumerate(zip(self.n_old, self.n_new)):
            assert torch.all(self.out[b, m:] == 7.0) and torch.all(self.lse[b, m:] == 7.0), "padding was written"
            if m == 0 or b in skip:
                continue
            r = held.attention(self.q[b], self.K[b], self.V[b], a + m, m, self.masks[b], 1.0 / math.sqrt(self.d))
            for name, got in (("out", self.out[b, :m]), ("lse", self.lse[b, :m])):
                worst[name] = max(worst.get(name, 0.0), plain.check(got, r[name], r[name + "_tol"], "%s[%d]" % (name, b)))
        print(worst)
        return self


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", SHAPES)
def test_attend(B, kind, Hq, Hkv, d, n_old, n_new):
    x = Draft(B, kind, Hq, Hkv, d, n_old, n_new)
    before = [t.clone() for t in (x.c.K, x.c.V, x.c.S, x.c.pos, x.c.seq_len, x.c.next_pos)]
    x.attend().check()
    for t, u in zip(before, (x.c.K, x.c.V, x.c.S, x.c.pos, x.c.seq_len, x.c.next_pos)):
        assert torch.equal(t, u)
    assert int(x.c.status.item()) == 0


MANY = [  # as many units as it takes for workgroups of 64 and of 128 rows, in groups of waves and not
    (16, 8, 128, [0, 1, 31, 32, 33, 63, 64, 65, 96, 97] * 2, [30, 30, 1, 29, 0, 17, 32, 30, 16, 30] * 2),
    (28, 4, 128, [0, 300, 64, 95] * 4, [30, 30, 11, 0] * 4),
    (16, 8, 64, [2100, 0, 1, 130] * 4, [64, 64, 33, 5] * 4),
    (16, 8, 64, [0, 33, 64, 190] * 2, [150, 149, 64, 1] * 2),
    (20, 10, 128, [0, 31, 64, 129] * 4, [130, 64, 129, 3] * 4),
]


@pytest.mark.parametrize("kind", ["dense", "paged", "e4m3", "int8_paged"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", MANY)
def test_attend_many_units(B, kind, Hq, Hkv, d, n_old, n_new):
    Draft(B, kind, Hq, Hkv, d, n_old, n_new, how="deep" if d == 64 else "any", seed=7).attend().check()


@pytest.mark.parametrize("kind", ["dense", "paged", "e4m3", "int8_paged"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", [(8, 1, 128, [2100, 10, 700], [2, 1, 0]), (8, 1, 128, [2100, 10], [20, 4]), (8, 1, 64, [1, 1600], [3, 9]),
                                                  (16, 1, 128, [1600, 50, 0, 1], [131, 130, 131, 1])])
def test_attend_two_to_four_shares(B, kind, Hq, Hkv, d, n_old, n_new):
    Draft(B, kind, Hq, Hkv, d, n_old, n_new, seed=8).attend().check()


@pytest.mark.parametrize("kind", ["dense", "int8_paged"])
@pytest.mark.parametrize("how", ["flat", "deep"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", [SHAPES[1], SHAPES[5], SHAPES[7], SHAPES[8]])
def test_attend_other_trees(B, kind, how, Hq, Hkv, d, n_old, n_new):
    Draft(B, kind, Hq, Hkv, d, n_old, n_new, how=how, seed=3).attend().check()


@pytest.mark.parametrize("kind", ["dense", "paged", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", [SHAPES[0], SHAPES[1], SHAPES[6], SHAPES[7], SHAPES[8]])
def test_a_chain_is_a_chunk(B, kind, Hq, Hkv, d, n_old, n_new):
    """Tokens that follow each other: what dynts_chunk_attend gives, either within its bound of the definition."""
    x = Draft(B, kind, Hq, Hkv, d, n_old, n_new, how="chain").attend()
    out, lse = torch.full_like(x.out, 7.0), torch.full_like(x.lse, 7.0)
    B.dynts_chunk_attend(x.c.ctx, 0, x.q.to(DEV), out, x.scratch, lse=lse, n_new=x.n)
    for b, (a, m) in enumerate(zip(n_old, n_new)):
        if m:
            r = held.attention(x.q[b], x.K[b], x.V[b], a + m, m, x.masks[b], 1.0 / math.sqrt(d))
            plain.check(out[b, :m], x.out[b, :m].double().cpu(), 2 * r["out_tol"], "out")
            plain.check(lse[b, :m], x.lse[b, :m].double().cpu(), 2 * r["lse_tol"], "lse")


@pytest.mark.parametrize("kind", ["dense", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", [SHAPES[1], SHAPES[3], SHAPES[7], SHAPES[8], (4, 4, 64, [0, 0], [70, 1])])
def test_any_pattern(B, kind, Hq, Hkv, d, n_old, n_new):
    """Tokens that see some of those behind them, not themselves, or nothing; bits behind the sequence's last count as 0."""
    def some(gen, m):
        x = torch.rand((m, m), generator=gen) < 0.3
        x[::4] = False
        return x
    x = Draft(B, kind, Hq, Hkv, d, n_old, n_new, masks=some)
    T, W = x.T, x.seen.shape[-1]
    for b, m in enumerate(n_new):
        behind = torch.zeros((T, T), dtype=torch.bool)
        behind[:, m:] = True
        x.seen[b] |= held.words(behind, T).to(DEV)
        if T % 32:
            x.seen[b, :, W - 1] |= -(1 << (T % 32)) if T % 32 < 31 else -(1 << 31)
    x.attend().check()
    for b, (a, m) in enumerate(zip(n_old, n_new)):
        if a == 0 and m:
            assert torch.all(x.out[b, 0:m:4] == 0) and torch.all(x.lse[b, 0:m:4] == -math.inf)


def test_hidden_rows_may_hold_anything(B):
    """K rows that a token does not see may hold NaN: the tokens that do not see them are not touched by them."""
    for many in (False, True):
        x = Draft(B, "dense", 8, 2, 64, [70], [600 if many else 8], how="flat")
        x.c.K[0, :, :, 73] = math.nan
        x.attend()
        x.out[0, 3], x.lse[0, 3] = 7.0, 7.0
        x.K[0, :, 73] = 0
        for i in range(x.n_new[0]):
            x.masks[0][i, 3] = False
        r = held.attention(x.q[0], x.K[0], x.V[0], 70 + x.n_new[0], x.n_new[0], x.masks[0], 1 / 8.0)
        rest = [i for i in range(x.n_new[0]) if i != 3]
        plain.check(x.out[0, rest], r["out"][rest], r["out_tol"][rest], "out")


# ---- step and keep -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("external", [False, True])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", [SHAPES[0], SHAPES[1], SHAPES[4], SHAPES[7], (8, 2, 64, [0, 63, 64, 500], [200, 130, 70, 129])])
def test_step_and_keep(B, kind, Hq, Hkv, d, n_old, n_new, external):
    """A draft appended and attended, its accepted path kept, the scores of it: the cache of a chain of the same tokens."""
    x = Draft(B, kind, Hq, Hkv, d, n_old, n_new, how="deep" if d == 64 else "any", append=False, external=external, L=2)
    Nb, T, c = len(n_old), x.T, x.c
    for b, a in enumerate(n_old):  # gaps in the positions, scores of the cached tokens
        c.pos[1, b, :, :a] = torch.arange(a, dtype=torch.int32, device=DEV) * 2
        c.next_pos[1, b] = 3 * a + 1
        if not external:
            c.S[1, b, :, :a] = torch.rand((Hkv, a), generator=x.gen).to(DEV)
    other = [c.K[0].clone(), c.S[0].clone(), c.seq_len[0].clone()]
    S0 = c.S[1].clone()
    taken = torch.full((Nb,), 99, dtype=torch.int32, device=DEV)
    x.step(taken, layer=1).check()
    assert taken.tolist() == n_new and c.seq_len[1].tolist() == [a + m for a, m in zip(n_old, n_new)]
    leaf = [m - 1 if b % 3 == 0 else int(torch.randint(-1, m, (1,), generator=x.gen)) if m else -1 for b, m in enumerate(n_new)]
    kept = torch.full((Nb,), 99, dtype=torch.int32, device=DEV)
    q_kept, lse_kept = torch.full_like(x.out, 5.0), torch.full_like(x.lse, 5.0)
    q = x.q.to(DEV)
    B.dynts_tree_keep(c.ctx, 1, x.seen, _ints(leaf), taken, kept, q=q, lse=x.lse, q_kept=q_kept, lse_kept=lse_kept)
    paths = [x.masks[b][i].nonzero().flatten().tolist() if i >= 0 else [] for b, i in enumerate(leaf)]
    assert kept.tolist() == [len(p) for p in paths]
    assert c.seq_len[1].tolist() == [a + len(p) for a, p in zip(n_old, paths)]
    assert c.next_pos[1].tolist() == [3 * a + 1 + len(p) for a, p in zip(n_old, paths)]
    K, V = c.K[1], c.V[1]
    for b, (a, p) in enumerate(zip(n_old, paths)):
        rows, n = list(range(a)) + [a + i for i in p], a + len(p)
        assert torch.equal(K[b, :, :n].double().cpu(), x.K[b][:, rows]) and torch.equal(V[b, :, :n].double().cpu(), x.V[b][:, rows])
        pos = torch.cat((torch.arange(a) * 2, 3 * a + 1 + torch.arange(len(p)))).to(torch.int32)
        assert torch.equal(c.pos[1, b, :, :n].cpu(), pos.expand(Hkv, n))
        want = x.s[b].t()[:, rows] if external else torch.cat((S0[b, :, :a].cpu(), torch.zeros(Hkv, len(p))), dim=1)
        assert torch.equal(c.S[1, b, :, :n].cpu(), want)
        assert torch.equal(q_kept[b, :len(p)], q[b, p]) and torch.equal(lse_kept[b, :len(p)], x.lse[b, p])
        assert torch.all(q_kept[b, len(p):] == 5.0) and torch.all(lse_kept[b, len(p):] == 5.0)
    dst = torch.zeros((Nb, Hkv, x.cap), dtype=torch.float32, device=DEV)
    B.dynts_chunk_scores(c.ctx, 1, q_kept, lse_kept, dst=dst, accumulate=False, n_new=kept)
    for b, (a, p) in enumerate(zip(n_old, paths)):
        if p:
            rows, n = list(range(a)) + [a + i for i in p], a + len(p)
            r = plain.attention(x.q[b, p], x.K[b][:, rows], x.V[b][:, rows], torch.arange(n).expand(Hkv, n), n, len(p), 1 / math.sqrt(d))
            # (the lse of the draft in place of the chain's own: the same sum in another order, both within lse_tol)
            tol = r["recv_tol"] + 2 * float(r["lse_tol"].max()) * r["recv"]
            plain.check(dst[b, :, :n], r["recv"], tol, "received[%d]" % b)
    # (the other layer's slots: behind its lengths a paged cache has none)
    assert torch.equal(other[1], c.S[0]) and torch.equal(other[2], c.seq_len[0])
    assert all(torch.equal(other[0][b, :, :a], c.K[0][b, :, :a]) for b, a in enumerate(n_old))
    assert int(c.status.item()) == 0
    if "paged" in kind:
        assert len(set(c.pages_in_use())) == 1


@pytest.mark.parametrize("kind", ["dense", "paged", "int8_paged"])
def test_keep_whole_chains_and_long_drafts(B, kind):
    """4096 drafted tokens: all of a chain stay, every second of a pair of chains, one, none; nothing else gathered."""
    Nb, T, Hkv, d = 4, 4096, 2, 64
    x = Draft(B, kind, 2, Hkv, d, [3, 60, 0, 129], [T, T, T, T], how="chain", append=False)
    parents = [x.parents[0], [i - 2 if i > 1 else -1 for i in range(T)], x.parents[2], x.parents[3]]
    B.dynts_tree_build(_ints(parents), x.seen)
    taken, kept = torch.zeros((Nb,), dtype=torch.int32, device=DEV), torch.zeros((Nb,), dtype=torch.int32, device=DEV)
    x.step(taken)
    leaf = [T - 1, T - 1, 0, -1]
    B.dynts_tree_keep(x.c.ctx, 0, x.seen, _ints(leaf), taken, kept)
    assert kept.tolist() == [T, T // 2, 1, 0] and x.c.seq_len[0].tolist() == [3 + T, 60 + T // 2, 1, 129]
    K, V = x.c.K[0], x.c.V[0]
    for b, rows in enumerate([list(range(3 + T)), list(range(60)) + [60 + i for i in range(1, T, 2)], [0], list(range(129))]):
        assert torch.equal(K[b, :, :len(rows)].double().cpu(), x.K[b][:, rows]) and torch.equal(V[b, :, :len(rows)].double().cpu(), x.V[b][:, rows])
    if "paged" in kind:
        assert len(set(x.c.pages_in_use())) == 1


def test_leaves_that_are_none(B):
    """A leaf outside its draft keeps nothing and is told of; n_taken may be left out."""
    x = Draft(B, "paged", 8, 2, 64, [10, 70, 5, 0], [6, 6, 6, 6], append=False)
    taken, kept = torch.zeros((4,), dtype=torch.int32, device=DEV), torch.full((4,), 99, dtype=torch.int32, device=DEV)
    x.step(taken)
    B.dynts_tree_keep(x.c.ctx, 0, x.seen, _ints([6, -2, 2 ** 31 - 1, -(2 ** 31)]), None, kept, q=x.q.to(DEV), lse=x.lse, q_kept=torch.zeros_like(x.out),
                      lse_kept=torch.zeros_like(x.lse))
    assert kept.tolist() == [0, 0, 0, 0] and x.c.seq_len[0].tolist() == [10, 70, 5, 0] and int(x.c.status.item()) == 16
    assert len(set(x.c.pages_in_use())) == 1


@pytest.mark.parametrize("kind", ["dense", "paged", "e4m3_paged"])
def test_drafts_that_do_not_fit(B, kind):
    """A draft without room leaves its sequence alone, also when a leaf of it is accepted."""
    kw = dict(n_pages=2 * 4 + 2) if "paged" in kind else {}
    x = Draft(B, kind, 8, 2, 64, [60, 40, 60], [30, 9, 64], append=False, spare=0, short=4, **kw)  # capacity 120: the last draft does not fit
    rows = x.c.K.clone()
    taken, kept = torch.zeros((3,), dtype=torch.int32, device=DEV), torch.full((3,), 99, dtype=torch.int32, device=DEV)
    x.step(taken)
    assert taken.tolist() == [30, 9, 0] and x.c.seq_len[0].tolist() == [90, 49, 60] and int(x.c.status.item()) == 1
    assert torch.all(x.out[2] == 7.0)
    x.c.status.zero_()
    B.dynts_tree_keep(x.c.ctx, 0, x.seen, _ints([29, -1, 63]), taken, kept)
    assert kept.tolist()[1:] == [0, 0] and x.c.seq_len[0].tolist()[1:] == [40, 60] and int(x.c.status.item()) == 16
    assert torch.equal(x.c.K[0, 2, :, :60], rows[0, 2, :, :60]) and torch.equal(x.c.K[0, 1, :, :40], rows[0, 1, :, :40])
    if "paged" in kind:
        assert len(set(x.c.pages_in_use())) == 1


@pytest.mark.parametrize("kind", ["dense", "paged"])
def test_drafts_among_single_steps(B, kind):
    """Single steps, whose score update is owed, between drafts: lengths, rows, outputs and scores of a cache that saw the accepted tokens alone, one by one."""
    gen = torch.Generator().manual_seed(21)
    Nb, Hq, Hkv, d, T = 2, 8, 2, 128, 11
    mk = lambda: _cache(B, kind, Nb, Hq, Hkv, d, 200)
    a, b = mk(), mk()
    K0, V0, m0 = _rand(gen, Nb, Hkv, 10, d).to(DEV), _rand(gen, Nb, Hkv, 10, d).to(DEV), _ints([10, 7])
    for c in (a, b):
        B.dynts_prefill(c.ctx, 0, K0, V0, m0)
    scratch = torch.empty(B.dynts_chunk_scratch_bytes(a.cfg, T), dtype=torch.uint8, device=DEV)
    seen, taken, kept = (torch.zeros(s, dtype=torch.int32, device=DEV) for s in ((Nb, T, 1), (Nb,), (Nb,)))
    o1, o2 = (torch.zeros((Nb, Hq, d), dtype=torch.float32, device=DEV) for _ in range(2))
    for turn in range(4):
        for _ in range(3):
            q, k, v = _rand(gen, Nb, Hq, d).to(DEV), _rand(gen, Nb, Hkv, d).to(DEV), _rand(gen, Nb, Hkv, d).to(DEV)
            B.dynts_decode_step(a.ctx, 0, q, k, v, o1)
            B.dynts_decode_step(b.ctx, 0, q, k, v, o2)
            # (the drafts' weights are the only thing rounded otherwise, and they stay out of K and V)
            assert torch.allclose(o1, o2, rtol=0, atol=1e-5)
        parents = [_parents(gen, T, "any") for _ in range(Nb)]
        masks = [held.ancestors(p, T)[0] for p in parents]
        q, k, v = _rand(gen, Nb, T, Hq, d).to(DEV), _rand(gen, Nb, T, Hkv, d).to(DEV), _rand(gen, Nb, T, Hkv, d).to(DEV)
        out, lse = torch.zeros((Nb, T, Hq, d), dtype=torch.bfloat16, device=DEV), torch.zeros((Nb, T, Hq), dtype=torch.float32, device=DEV)
        qk, lk = torch.zeros_like(out), torch.zeros_like(lse)
        B.dynts_tree_build(_ints(parents), seen)
        B.dynts_tree_step(a.ctx, 0, q, k, v, seen, taken, out, scratch, lse=lse)
        B.dynts_tree_keep(a.ctx, 0, seen, _ints([T - 1, T - 2]), taken, kept, q=q, lse=lse, q_kept=qk, lse_kept=lk)
        B.dynts_chunk_scores(a.ctx, 0, qk, lk, n_new=kept)
        paths = [masks[i][leaf].nonzero().flatten().tolist() for i, leaf in enumerate((T - 1, T - 2))]
        for step in range(max(map(len, paths))):
            at = [p[step] if step < len(p) else 0 for p in paths]
            active = torch.tensor([step < len(p) for p in paths], dtype=torch.uint8, device=DEV)
            row = lambda x: torch.stack([x[i, at[i]] for i in range(Nb)]).contiguous()
            B.dynts_decode_step(b.ctx, 0, row(q), row(k), row(v), o2, active=active)
            for i, p in enumerate(paths):
                if step < len(p):
                    assert (o2[i] - out[i, p[step]].float()).abs().max() <= 6 * 2.0 ** -7
    for c in (a, b):
        B.dynts_update_scores(c.ctx, 0)
    assert torch.equal(a.seq_len, b.seq_len) and torch.equal(a.next_pos, b.next_pos)
    Ka, Va, Kb, Vb = a.K[0], a.V[0], b.K[0], b.V[0]
    for i, n in enumerate(a.seq_len[0].tolist()):
        assert torch.equal(Ka[i, :, :n], Kb[i, :, :n]) and torch.equal(Va[i, :, :n], Vb[i, :, :n]) and torch.equal(a.pos[0, i, :, :n], b.pos[0, i, :, :n])
        fin = torch.isfinite(b.S[0, i, :, :n])
        assert torch.allclose(a.S[0, i, :, :n][fin], b.S[0, i, :, :n][fin], rtol=0, atol=1e-4)


@pytest.mark.parametrize("kind", ["paged", "e4m3"])
def test_recorded_drafts(B, kind):
    """Build, step, keep and scores recorded as one graph and replayed with other drafts, eager work between: as eager calls on a cache beside it."""
    gen = torch.Generator().manual_seed(23)
    Nb, Hq, Hkv, d, T = 6, 28, 4, 128, 40
    caches = [_cache(B, kind, Nb, Hq, Hkv, d, 600) for _ in range(2)]
    scratch = torch.empty(B.dynts_codes_scratch_bytes(caches[0].cfg, T), dtype=torch.uint8, device=DEV)
    inp = dict(q=torch.zeros((Nb, T, Hq, d), dtype=torch.bfloat16, device=DEV), k=torch.zeros((Nb, T, Hkv, d), dtype=torch.bfloat16, device=DEV),
               v=torch.zeros((Nb, T, Hkv, d), dtype=torch.bfloat16, device=DEV), parents=torch.full((Nb, T), -1, dtype=torch.int32, device=DEV),
               leaf=torch.zeros((Nb,), dtype=torch.int32, device=DEV))
    bufs = [dict(seen=torch.zeros((Nb, T, 2), dtype=torch.int32, device=DEV), taken=torch.zeros((Nb,), dtype=torch.int32, device=DEV),
                 kept=torch.zeros((Nb,), dtype=torch.int32, device=DEV), out=torch.zeros_like(inp["q"]), qk=torch.zeros_like(inp["q"]),
                 lse=torch.zeros((Nb, T, Hq), dtype=torch.float32, device=DEV), lk=torch.zeros((Nb, T, Hq), dtype=torch.float32, device=DEV)) for _ in range(2)]

    def draft(c, o):
        B.dynts_tree_build(inp["parents"], o["seen"])
        B.dynts_tree_step(c.ctx, 0, inp["q"], inp["k"], inp["v"], o["seen"], o["taken"], o["out"], scratch, lse=o["lse"])
        B.dynts_tree_keep(c.ctx, 0, o["seen"], inp["leaf"], o["taken"], o["kept"], q=inp["q"], lse=o["lse"], q_kept=o["qk"], lse_kept=o["lk"])
        B.dynts_chunk_scores(c.ctx, 0, o["qk"], o["lk"], n_new=o["kept"])

    for c, o in zip(caches, bufs):
        draft(c, o)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        draft(caches[0], bufs[0])
    for turn in range(4):
        for k in "qkv":
            inp[k].copy_(_rand(gen, *inp[k].shape))
        inp["parents"].copy_(torch.tensor([_parents(gen, T, "deep" if turn % 2 else "any") for _ in range(Nb)], dtype=torch.int32))
        inp["leaf"].copy_(torch.randint(-1, T, (Nb,), generator=gen).to(torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        draft(caches[1], bufs[1])
        for k in bufs[0]:
            assert torch.equal(bufs[0][k], bufs[1][k]), k
        assert torch.equal(caches[0].S, caches[1].S) and torch.equal(caches[0].seq_len, caches[1].seq_len)
        torch.cuda.synchronize()
    n = caches[0].seq_len[0].tolist()
    assert max(n) > 20 and int(caches[0].status.item()) == 0
    Ka, Kb = caches[0].K[0], caches[1].K[0]
    assert all(torch.equal(Ka[i, :, :m], Kb[i, :, :m]) for i, m in enumerate(n))
