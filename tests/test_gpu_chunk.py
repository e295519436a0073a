"""Chunks of new tokens (dynts_chunk_*) against the definition in float64 and against single steps."""
import math

import numpy as np
import pytest
import torch

from tests import chunk_plain as plain
from tests.helpers import f64

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def B():
    from paper_2601_18383_amd import binding
    return binding


def _rand(gen, *shape, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(torch.bfloat16)


def _positions(gen, Hkv, n_old, m, gaps):
    """[Hkv][n_old + m]: ascending, with `gaps` positions missing among the cached ones (elsewhere in every head)."""
    extra = torch.floor(torch.rand((Hkv, n_old), generator=gen).sort(dim=-1).values * (gaps + 1))
    return torch.cat((torch.arange(n_old) + extra, (n_old + gaps + torch.arange(m)).expand(Hkv, m)), dim=1).to(torch.int32)


class Case:
    """A cache of several sequences with n_old slots and chunks of n_new tokens, on the CPU and (fill) on the device."""

    def __init__(self, B, layout, Hq, Hkv, d, n_old, n_new, T=None, gaps=0, seed=0, spare=5, external=False, qscale=1.0):
        self.gen = gen = torch.Generator().manual_seed(seed + 7 * d + Hq)
        self.B, self.Hq, self.Hkv, self.d = B, Hq, Hkv, d
        self.n_old, self.n_new, Nb = n_old, n_new, len(n_old)
        self.T = T = T or max(max(n_new), 1)
        self.cap = max(a + b for a, b in zip(n_old, n_new)) + spare
        self.K = _rand(gen, Nb, Hkv, self.cap, d)
        self.V = _rand(gen, Nb, Hkv, self.cap, d)
        self.q = _rand(gen, Nb, T, Hq, d, scale=qscale)
        self.pos = [_positions(gen, Hkv, a, b, gaps) for a, b in zip(n_old, n_new)]
        self.next = [a + gaps for a in n_old]
        kw = dict(external_scores=external)
        self.cache = (B.Cache if layout == "dense" else B.PagedCache)(1, Nb, Hq, Hkv, d, self.cap, 0, 0, 1, **kw)
        self.scratch = torch.empty(B.dynts_chunk_scratch_bytes(self.cache.cfg, T), dtype=torch.uint8, device=DEV)
        self.scratch.fill_(0xA5)
        self.n = torch.tensor(n_new, dtype=torch.int32, device=DEV)
        self.out = torch.full((Nb, T, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((Nb, T, Hq), 7.0, dtype=torch.float32, device=DEV)
        pad = lambda x: torch.stack([torch.cat((x[b, :, a:a + m].transpose(0, 1), torch.full((T - m, Hkv, d), math.nan, dtype=x.dtype)))
                                     for b, (a, m) in enumerate(zip(n_old, n_new))]).contiguous().to(DEV)
        self.k_new, self.v_new = pad(self.K), pad(self.V)       # rows behind a chunk are NaN
        for b, m in enumerate(n_new):
            self.q[b, m:] = math.nan

    def fill(self, chunk_too):
        """The cached rows (and the chunk's, if it is not to be appended) by way of dynts_prefill, then as thinking tokens."""
        c = self.cache
        lens = [a + (m if chunk_too else 0) for a, m in zip(self.n_old, self.n_new)]
        self.B.dynts_prefill(c.ctx, 0, self.K.to(DEV), self.V.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV))
        c.n_prompt.zero_()
        c.S.zero_()
        for b, n in enumerate(lens):
            c.pos[0, b, :, :n] = self.pos[b][:, :n].to(DEV)
            c.next_pos[0, b] = self.next[b] + (self.n_new[b] if chunk_too else 0)
        return self

    def check(self, what="", lse=None, recv=None, **shape):
        """out (and lse, recv) against the definition; padding untouched."""
        per = {k: shape.pop(k, None) for k in ("first", "last")}
        scale = shape.pop("scale", 1.0 / math.sqrt(self.d))
        worst = {}
        for b, (a, m) in enumerate(zip(self.n_old, self.n_new)):
            assert torch.all(self.out[b, m:] == 7.0), "padding of sequence %d was written" % b
            if lse is not None:
                assert torch.all(lse[b, m:] == 7.0)
            if m == 0:
                continue
            kw = dict(shape, **{k: (v[b] if v is not None else None) for k, v in per.items()})
            r = plain.attention(self.q[b], self.K[b], self.V[b], self.pos[b], a + m, m, scale, **kw)
            name = "%s[%d]" % (what, b)
            worst["out"] = max(worst.get("out", 0), plain.check(self.out[b, :m], r["out"], r["out_tol"], name + " out"))
            if lse is not None:
                worst["lse"] = max(worst.get("lse", 0), plain.check(lse[b, :m], r["lse"], r["lse_tol"], name + " lse"))
            if recv is not None:
                worst["recv"] = max(worst.get("recv", 0), plain.check(recv[b, :, :a + m], r["recv"], r["recv_tol"], name + " received"))
        print(what, worst)
        return worst


SHAPES = [  # Hq, Hkv, d, n_old, n_new
    (8, 2, 64, [0, 1, 63, 64, 200, 129], [1, 1, 1, 1, 1, 1]),           # single tokens, lengths around a page
    (28, 4, 128, [0, 5, 300, 64], [37, 0, 12, 64]),                     # odd groups, an empty chunk, an empty cache
    (6, 6, 128, [130, 77], [33, 65]),                                   # no sharing of KV heads
    (16, 1, 64, [500, 3], [9, 100]),                                    # the largest group
    (16, 1, 128, [40], [257]),
    (32, 8, 128, [1000], [16]),
    (4, 2, 64, [10, 700], [300, 129]),                                  # several row blocks
    (8, 2, 128, [2500, 1], [5, 2]),
    (8, 1, 128, [3000, 10], [200, 64]),                                 # keys in shares; a short cache beside it
    (4, 1, 64, [4000, 900], [300, 1]),
    (28, 4, 128, [0, 31, 32, 33, 100, 257, 64, 1, 5, 0, 90, 128], [60, 60, 1, 59, 0, 33, 60, 37, 32, 31, 64, 7]),  # many rows of many units
    (16, 8, 64, [0, 1, 63, 64, 65, 200, 31, 0] * 2, [150, 149, 64, 1, 0, 128, 65, 150] * 2),
    (8, 2, 128, [8000], [600]),                                         # many rows of few units: keys in shares
    (8, 2, 64, [3500], [600]),
    (16, 1, 128, [50, 0, 7] * 4, [70, 65, 8] * 4),                      # the largest group, many rows
    (32, 8, 128, [700, 0, 300, 64, 10, 650], [100, 99, 64, 130, 1, 33]),  # many slots of many units, several groups of rows
]
MANY = SHAPES[10:]


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", SHAPES)
def test_attend_and_scores(B, layout, Hq, Hkv, d, n_old, n_new):
    c = Case(B, layout, Hq, Hkv, d, n_old, n_new, gaps=50, qscale=2.0).fill(True)
    dst = torch.full((len(n_old), Hkv, c.cap), 7.0, dtype=torch.float32, device=DEV)
    before = [t.clone() for t in (c.cache.K, c.cache.V, c.cache.S, c.cache.pos, c.cache.seq_len, c.cache.next_pos)]
    q = c.q.to(DEV)
    B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n)
    B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n)
    c.check("plain", lse=c.lse, recv=dst)
    for b, (a, m) in enumerate(zip(n_old, n_new)):
        assert torch.all(dst[b, :, (a + m if m else 0):] == 7.0), "slots beyond the length were written"
    once = dst.clone()
    B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, n_new=c.n)  # the same again on top
    for b, (a, m) in enumerate(zip(n_old, n_new)):
        if m:
            assert torch.equal(dst[b, :, :a + m], 2 * once[b, :, :a + m])
    for t, u in zip(before, (c.cache.K, c.cache.V, c.cache.S, c.cache.pos, c.cache.seq_len, c.cache.next_pos)):
        assert torch.equal(t, u)
    # without lse, and with the padding's length given as the chunk's: the same outputs
    again = torch.full_like(c.out, 7.0)
    B.dynts_chunk_attend(c.cache.ctx, 0, q, again, c.scratch, n_new=c.n)
    assert torch.equal(again, c.out)
    assert int(c.cache.status.item()) == 0


def _shapings(c, gen, kind):
    """Shaping tensors for a case, on the CPU: dict of softcap, window, slope, first, last."""
    Nb, T = len(c.n_old), c.T
    own = torch.stack([c.next[b] + torch.arange(T) for b in range(Nb)]).to(torch.int32)
    s = {}
    if "cap" in kind:
        s["softcap"] = 3.0 if "tight" in kind else 30.0
    if "slope" in kind:
        s["slope"] = (2.0 ** (-8.0 * (1 + torch.arange(c.Hq)) / c.Hq)).to(torch.float32)
    if "window" in kind:
        s["window"] = 1 if "one" in kind else 40
    if "documents" in kind:  # starts every few positions
        s["first"] = (own // 23 * 23).to(torch.int32)
    if "prefix" in kind:
        edge = own[:, :1] + T // 2
        s["last"] = torch.where(own <= edge, edge.expand_as(own), own).to(torch.int32)
    if "empty" in kind:  # rows that see nothing: an interval that ends before it begins, one before and one behind the cache
        first = s.get("first", torch.zeros_like(own)).clone()
        last = s.get("last", own.clone())
        first[:, ::3], last[:, ::3] = 10, 9
        first[:, 1::5], last[:, 1::5] = 1 << 30, (1 << 30) + 5
        last[:, 2::7] = -4
        s["first"], s["last"] = first, last
    if "future" in kind:  # everybody sees everything, the keys behind them too
        s["last"] = torch.full_like(own, (1 << 31) - 1)
    return s


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("kind", ["cap", "cap_tight", "slope", "window", "window_one", "documents", "prefix", "empty", "future",
                                  "cap_slope_window_documents_prefix", "slope_prefix_empty"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", [SHAPES[0], SHAPES[1], SHAPES[3], SHAPES[6], SHAPES[7], SHAPES[9]] + MANY)
def test_shaped(B, layout, kind, Hq, Hkv, d, n_old, n_new):
    c = Case(B, layout, Hq, Hkv, d, n_old, n_new, gaps=90, seed=11, qscale=2.0).fill(True)
    s = _shapings(c, c.gen, kind)
    on = {k: (v.to(DEV) if torch.is_tensor(v) else v) for k, v in s.items()}
    sh = B.Shaping(**on)
    dst = torch.full((len(n_old), Hkv, c.cap), 7.0, dtype=torch.float32, device=DEV)
    q = c.q.to(DEV)
    B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n, shaping=sh)
    B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n, shaping=sh)
    c.check(kind, lse=c.lse, recv=dst, **s)
    if "empty" in kind:
        m = c.n_new[0]
        assert torch.all(c.out[0, :m:3] == 0) and torch.all(c.lse[0, :m:3] == -math.inf)
    assert int(c.cache.status.item()) == 0


@pytest.mark.parametrize("kind", ["slope", "window", "documents", "prefix", "empty", "future", "cap_slope_window_documents_prefix", "slope_prefix_empty"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", [SHAPES[1], SHAPES[7], SHAPES[9], (8, 2, 128, [300, 0, 1], [500, 400, 31]), (8, 2, 64, [0, 70], [600, 450])])
def test_shaped_without_gaps(B, kind, Hq, Hkv, d, n_old, n_new):
    """Positions that go up by one, from 17 on: slots are found without a search, and the bias of a tile is linear."""
    c = Case(B, "dense", Hq, Hkv, d, n_old, n_new, seed=13, qscale=2.0)
    c.pos, c.next = [p + 17 for p in c.pos], [p + 17 for p in c.next]
    c.fill(True)
    s = _shapings(c, c.gen, kind)
    sh = B.Shaping(**{k: (v.to(DEV) if torch.is_tensor(v) else v) for k, v in s.items()})
    dst = torch.full((len(n_old), Hkv, c.cap), 7.0, dtype=torch.float32, device=DEV)
    q = c.q.to(DEV)
    B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n, shaping=sh)
    B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n, shaping=sh)
    c.check(kind, lse=c.lse, recv=dst, **s)


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("missing", [1, 3, 5])
def test_gaps_that_make_up_for_a_short_tile(B, layout, missing):
    """The last tile has 29 slots, whose positions span 29 + missing: with 3 as many as a whole tile without gaps."""
    c = Case(B, layout, 32, 2, 128, [54] * 33, [7] * 33, seed=17, qscale=0.5)
    for b in range(33):
        c.pos[b] = c.pos[b] + missing * (torch.arange(61) >= 40).to(torch.int32)
    c.next = [n + missing for n in c.next]
    c.fill(True)
    s = _shapings(c, c.gen, "slope")
    sh = B.Shaping(slope=s["slope"].to(DEV))
    dst = torch.full((33, 2, c.cap), 7.0, dtype=torch.float32, device=DEV)
    q = c.q.to(DEV)
    B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n, shaping=sh)
    B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n, shaping=sh)
    c.check("slope", lse=c.lse, recv=dst, **s)


def test_keys_hidden_from_all_may_be_anything(B):
    """K rows of another document that hold NaN and infinities, and what lies behind the length in the cache."""
    c = Case(B, "dense", 8, 2, 64, [100], [70], seed=3).fill(True)
    c.cache.K[0, :, :, :40] = math.nan
    c.cache.K[0, :, :, 40:50] = math.inf
    c.cache.K[0, :, :, 170:] = math.nan
    c.cache.V[0, :, :, 170:] = math.nan
    first = torch.full((1, 70), 50, dtype=torch.int32)
    sh = B.Shaping(first=first.to(DEV))
    q = c.q.to(DEV)
    B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n, shaping=sh)
    dst = torch.zeros((1, 2, c.cap), dtype=torch.float32, device=DEV)
    B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n, shaping=sh)
    assert torch.all(dst[:, :, :50] == 0)
    c.K[:, :, :50] = 0
    c.check("hidden", lse=c.lse, recv=dst, first=first)


def test_a_scale_of_the_callers(B):
    c = Case(B, "dense", 8, 2, 64, [100, 3], [20, 40], seed=12)
    c.cache.close()
    c.cache = B.Cache(1, 2, 8, 2, 64, c.cap, 0, 0, 1, softmax_scale=0.31)
    c.fill(True)
    q = c.q.to(DEV)
    for shape in (dict(), dict(softcap=4.0), dict(softcap=4.0, window=30)):
        sh = B.Shaping(**shape) if shape else None
        dst = torch.zeros((2, 2, c.cap), dtype=torch.float32, device=DEV)
        B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n, shaping=sh)
        B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n, shaping=sh)
        c.check("scale", lse=c.lse, recv=dst, scale=0.31, **shape)


def test_late_and_large_maxima(B):
    """Keys that grow along the cache by hundreds of log2 units: every row's shift has to follow."""
    c = Case(B, "dense", 28, 4, 128, [1500, 0], [40, 200], seed=5, qscale=1.5)
    grow = torch.linspace(0, 1, c.cap)[None, None, :, None] * torch.tensor([30.0, 8.0])[:, None, None, None]
    c.K = (c.K.float() * (1 + grow)).to(torch.bfloat16)
    c.fill(True)
    q = c.q.to(DEV)
    B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n)
    dst = torch.zeros((2, 4, c.cap), dtype=torch.float32, device=DEV)
    B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n)
    c.check("growing", lse=c.lse, recv=dst)


# ---- the cache's state -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", [SHAPES[0], SHAPES[1], SHAPES[4], SHAPES[6]] + MANY)
def test_step_is_append_attend_scores(B, layout, Hq, Hkv, d, n_old, n_new):
    """One chunk: rows, positions, lengths and scores in the cache, outputs as the definition has them."""
    c = Case(B, layout, Hq, Hkv, d, n_old, n_new, gaps=20, seed=2).fill(False)
    c.cache.n_prompt.copy_(torch.tensor([min(4, a) for a in n_old], dtype=torch.int32))
    for b, a in enumerate(n_old):
        c.cache.S[0, b, :, :a] = torch.rand((Hkv, a), generator=c.gen).to(DEV)
        c.cache.S[0, b, :, :min(4, a)] = math.inf
    S0 = c.cache.S[0].clone()
    B.dynts_chunk_step(c.cache.ctx, 0, c.q.to(DEV), c.k_new, c.v_new, c.out, c.scratch, lse=c.lse, n_new=c.n)
    c.check("step", lse=c.lse)
    K, V = c.cache.K[0], c.cache.V[0]
    for b, (a, m) in enumerate(zip(n_old, n_new)):
        n, M = a + m, min(4, a)
        assert torch.equal(K[b, :, :n].cpu(), c.K[b, :, :n]) and torch.equal(V[b, :, :n].cpu(), c.V[b, :, :n])
        assert torch.equal(c.cache.pos[0, b, :, :n].cpu(), c.pos[b][:, :n])
        S = c.cache.S[0, b]
        assert torch.all(torch.isinf(S[:, :M])) and torch.equal(S[:, n:], S0[b, :, n:])
        if m:
            r = plain.attention(c.q[b], c.K[b], c.V[b], c.pos[b], n, m, 1.0 / math.sqrt(d))
            want = r["recv"].clone()
            want[:, :a] += S0[b, :, :a].double().cpu()
            plain.check(S[:, M:n], want[:, M:], r["recv_tol"][:, M:] + 2 * plain.HALF32 * want[:, M:].abs(), "S[%d]" % b)
    assert c.cache.seq_len[0].tolist() == [a + m for a, m in zip(n_old, n_new)]
    assert c.cache.next_pos[0].tolist() == [x + m for x, m in zip(c.next, n_new)]
    assert int(c.cache.status.item()) == 0
    if layout == "paged":
        used, taken = c.cache.pages_in_use()
        assert used == taken


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 64), (28, 4, 128)])
def test_chunks_among_single_steps_and_triggers(B, layout, Hq, Hkv, d):
    """Two caches go through the same tokens: one by single steps alone, the other in chunks between single steps, with owed
    score updates outstanding, and triggers.  Lengths, rows and positions agree bit for bit while selections do, outputs and scores
    within roundings."""
    gen = torch.Generator().manual_seed(9)
    Nb, M, budget, window, every = 2, 10, 40, 12, 30
    cap = M + budget + window + every + 40
    mk = lambda: (B.Cache if layout == "dense" else B.PagedCache)(1, Nb, Hq, Hkv, d, cap, budget, window, every)
    one, many = mk(), mk()
    K0, V0 = _rand(gen, Nb, Hkv, M, d).to(DEV), _rand(gen, Nb, Hkv, M, d).to(DEV)
    m = torch.full((Nb,), M, dtype=torch.int32, device=DEV)
    for c in (one, many):
        B.dynts_prefill(c.ctx, 0, K0, V0, m)
    scratch = torch.empty(B.dynts_chunk_scratch_bytes(one.cfg, 24), dtype=torch.uint8, device=DEV)
    o1 = torch.zeros((Nb, Hq, d), dtype=torch.float32, device=DEV)
    for turn, T in enumerate([1, 24, 7, 3, 16, 5, 24, 2]):
        q = _rand(gen, Nb, T, Hq, d).to(DEV)
        k, v = _rand(gen, Nb, T, Hkv, d).to(DEV), _rand(gen, Nb, T, Hkv, d).to(DEV)
        out = torch.zeros((Nb, T, Hq, d), dtype=torch.bfloat16, device=DEV)
        for i in range(T):
            B.dynts_decode_step(one.ctx, 0, q[:, i].contiguous(), k[:, i].contiguous(), v[:, i].contiguous(), o1)
            if turn % 3 == 2:  # these turns are single steps on either side, so that updates are owed when a chunk comes
                o2 = torch.zeros_like(o1)
                B.dynts_decode_step(many.ctx, 0, q[:, i].contiguous(), k[:, i].contiguous(), v[:, i].contiguous(), o2)
                assert torch.allclose(o1, o2, rtol=0, atol=1e-4)
            else:
                out_ref = o1.clone()
                if i == T - 1:
                    last = out_ref
        if turn % 3 != 2:
            B.dynts_chunk_step(many.ctx, 0, q, k, v, out, scratch)
            # (weights and outputs in bf16: half a step each of values of about 1)
            assert torch.allclose(out[:, -1].float(), last, rtol=2 ** -8, atol=2 ** -8 * 4)
        if int(one.seq_len[0, 0].item()) >= M + budget + window:
            for c in (one, many):
                B.dynts_select_evict(c.ctx, 0, c.keep_idx, c.new_len)
            assert torch.equal(one.new_len, many.new_len)
            n = int(one.new_len[0].item())
            many.keep_idx.copy_(one.keep_idx)  # (near ties may fall either way)
            for c in (one, many):
                B.dynts_compact(c.ctx, 0, c.keep_idx, c.new_len)
        for c in (one, many):
            B.dynts_update_scores(c.ctx, 0)
        n = int(one.seq_len[0, 0].item())
        assert torch.equal(one.seq_len, many.seq_len) and torch.equal(one.next_pos, many.next_pos)
        assert torch.equal(one.K[0][:, :, :n], many.K[0][:, :, :n]) and torch.equal(one.V[0][:, :, :n], many.V[0][:, :, :n])
        assert torch.equal(one.pos[0][:, :, :n], many.pos[0][:, :, :n])
        a, b = one.S[0][:, :, M:n], many.S[0][:, :, M:n]
        assert torch.allclose(a, b, rtol=1e-4, atol=1e-5), float((a - b).abs().max())
    assert int(one.status.item()) == 0 and int(many.status.item()) == 0


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 64), (28, 4, 128)])
@pytest.mark.parametrize("T", [3, 40])
@pytest.mark.parametrize("hinted", [False, True])
def test_a_chunk_while_an_update_is_owed(B, layout, Hq, Hkv, d, T, hinted):
    """A step's score update applied before a chunk, or behind it: by dynts_update_scores, by the next step, or by a trigger (for which the step
    may have kept its logits)."""
    gen = torch.Generator().manual_seed(21)
    Nb, M, n0 = 3, 8, 150
    cap = n0 + T + 4
    mk = lambda: (B.Cache if layout == "dense" else B.PagedCache)(1, Nb, Hq, Hkv, d, cap, 60, 10, 1)
    K0, V0 = _rand(gen, Nb, Hkv, n0, d).to(DEV), _rand(gen, Nb, Hkv, n0, d).to(DEV)
    q, k, v = (_rand(gen, Nb, T, h, d).to(DEV) for h in (Hq, Hkv, Hkv))
    qs, ks, vs = (_rand(gen, 2, Nb, h, d).to(DEV) for h in (Hq, Hkv, Hkv))

    def run(at_once, end):
        c = mk()
        B.dynts_prefill(c.ctx, 0, K0, V0, torch.full((Nb,), n0, dtype=torch.int32, device=DEV))
        c.n_prompt.fill_(M)
        c.S[:, :, :, M:] = 0
        o, out = torch.zeros((Nb, Hq, d), device=DEV), torch.zeros((Nb, T, Hq, d), dtype=torch.bfloat16, device=DEV)
        scratch = torch.empty(B.dynts_chunk_scratch_bytes(c.cfg, T), dtype=torch.uint8, device=DEV)
        if hinted:
            B.dynts_hint_trigger(c.ctx, 0)
        B.dynts_decode_step(c.ctx, 0, qs[0], ks[0], vs[0], o)
        if at_once:
            B.dynts_update_scores(c.ctx, 0)
        B.dynts_chunk_step(c.ctx, 0, q, k, v, out, scratch)
        if end == "step":
            B.dynts_decode_step(c.ctx, 0, qs[1], ks[1], vs[1], o)
        if end == "trigger":
            B.dynts_select_evict(c.ctx, 0, c.keep_idx, c.new_len)
        else:
            B.dynts_update_scores(c.ctx, 0)
        assert int(c.status.item()) == 0
        n = int(c.seq_len[0, 0].item())
        return c.S[0, :, :, :n].clone(), o, out

    for end in ("update", "step", "trigger"):
        (S, o, out), (S2, o2, out2) = run(True, end), run(False, end)
        assert torch.equal(out, out2) and torch.allclose(o, o2, rtol=0, atol=1e-5)
        assert torch.all(S[:, :, :M] == math.inf) and torch.all(S2[:, :, :M] == math.inf)
        # (two or three sums of numbers below G * T in another order: a half step each of what they add up to, and the weights of a step, formed
        # again from kept logits or K, a few half steps of theirs)
        assert torch.allclose(S[:, :, M:], S2[:, :, M:], rtol=2e-6, atol=2e-6), float((S[:, :, M:] - S2[:, :, M:]).abs().max())
        # mass: every row of the step, of the chunk and of the last step gives away what the question slots do not take
        assert float(S2[:, :, M:].sum()) > 0.5 * Nb * Hq * (T + 1)


@pytest.mark.parametrize("layout", ["dense", "paged"])
def test_question_in_chunks(B, layout):
    """A question in three chunks into an empty cache: the same cache as dynts_prefill leaves, and a question behind thinking
    tokens is refused."""
    gen = torch.Generator().manual_seed(4)
    Nb, Hq, Hkv, d, M = 3, 8, 2, 64, 150
    mk = lambda: (B.Cache if layout == "dense" else B.PagedCache)(2, Nb, Hq, Hkv, d, 400, 100, 20, 20)
    a, b = mk(), mk()
    K, V = _rand(gen, Nb, Hkv, M, d).to(DEV), _rand(gen, Nb, Hkv, M, d).to(DEV)
    q = _rand(gen, Nb, M, Hq, d).to(DEV)
    m = torch.full((Nb,), M, dtype=torch.int32, device=DEV)
    for layer in range(2):
        B.dynts_prefill(a.ctx, layer, K, V, m)
        scratch = torch.empty(B.dynts_chunk_scratch_bytes(b.cfg, 100), dtype=torch.uint8, device=DEV)
        outs = []
        for lo, hi in ((0, 100), (100, 101), (101, M)):
            k, v = (x[:, :, lo:hi].transpose(1, 2).contiguous() for x in (K, V))
            out = torch.zeros((Nb, hi - lo, Hq, d), dtype=torch.bfloat16, device=DEV)
            B.dynts_chunk_step(b.ctx, layer, q[:, lo:hi].contiguous(), k, v, out, scratch, question=True)
            outs.append(out)
    for name in ("S", "pos", "seq_len", "next_pos", "n_prompt"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    for name in ("K", "V"):  # (slots beyond the length belong to no page)
        assert torch.equal(getattr(a, name)[:, :, :, :M], getattr(b, name)[:, :, :, :M]), name
    assert int(b.status.item()) == 0
    whole = torch.zeros((Nb, M, Hq, d), dtype=torch.bfloat16, device=DEV)
    scratch = torch.empty(B.dynts_chunk_scratch_bytes(b.cfg, M), dtype=torch.uint8, device=DEV)
    B.dynts_chunk_attend(a.ctx, 0, q, whole, scratch)
    # (weights are rounded against another shift, so half a step of theirs and of the output's)
    assert torch.allclose(torch.cat(outs, 1).float(), whole.float(), rtol=2 ** -7, atol=2 ** -8 * 4)
    # a thinking token, then a question again
    one = lambda h: _rand(gen, Nb, 1, h, d).to(DEV)
    out = torch.full((Nb, 1, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    B.dynts_chunk_step(b.ctx, 0, one(Hq), one(Hkv), one(Hkv), out, scratch)
    n_new = torch.tensor([1, 0, 1], dtype=torch.int32, device=DEV)
    out.fill_(7.0)
    B.dynts_chunk_step(b.ctx, 0, one(Hq), one(Hkv), one(Hkv), out, scratch, n_new=n_new, question=True)
    assert int(b.status.item()) == 8
    assert torch.all(out == 7.0) and b.seq_len[0].tolist() == [M + 1] * Nb and b.n_prompt.tolist() == [M] * Nb


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("T", [6, 300])
def test_a_chunk_that_does_not_fit_leaves_its_sequence_alone(B, layout, T):
    c = Case(B, layout, 8, 2, 64, [20, 64, 0], [T, T, T], seed=8, spare=0)  # capacity 64 + T: the second just fits
    c.cache.close()
    cap = 63 + T
    c.cache = (B.Cache if layout == "dense" else B.PagedCache)(1, 3, 8, 2, 64, cap, 0, 0, 1)
    c.K, c.V = c.K[:, :, :cap], c.V[:, :, :cap]
    c.n_old = [20, 64, 0]
    c.fill(False)
    rows = 64 if layout == "paged" else cap  # (slots beyond the length belong to no page)
    state = lambda: [c.cache.K[0, 1, :, :rows], c.cache.V[0, 1, :, :rows], c.cache.S[0, 1], c.cache.pos[0, 1]]
    before = [t.clone() for t in state()]
    B.dynts_chunk_step(c.cache.ctx, 0, c.q.to(DEV), c.k_new, c.v_new, c.out, c.scratch, lse=c.lse, n_new=c.n)
    assert int(c.cache.status.item()) == 1
    assert c.cache.seq_len[0].tolist() == [20 + T, 64, T]
    assert torch.all(c.out[1] == 7.0) and torch.all(c.lse[1] == 7.0)
    for t, u in zip(before, state()):
        assert torch.equal(t, u)
    if layout == "paged":
        used, taken = c.cache.pages_in_use()
        assert used == taken


def test_a_pool_without_enough_pages(B):
    """Pages for one of two sequences: the other keeps what it had, and the pool its pages."""
    gen = torch.Generator().manual_seed(1)
    c = B.PagedCache(1, 2, 8, 2, 64, 400, 0, 0, 1, n_pages=9)
    K = _rand(gen, 2, 2, 64, 64).to(DEV)
    B.dynts_prefill(c.ctx, 0, K, K, torch.tensor([64, 64], dtype=torch.int32, device=DEV))  # four pages
    assert int(c.free_top.item()) == 5
    T = 70  # two more pages a head: four a sequence
    q, k = _rand(gen, 2, T, 8, 64).to(DEV), _rand(gen, 2, T, 2, 64).to(DEV)
    out = torch.full((2, T, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    scratch = torch.empty(B.dynts_chunk_scratch_bytes(c.cfg, T), dtype=torch.uint8, device=DEV)
    B.dynts_chunk_step(c.ctx, 0, q, k, k, out, scratch)
    assert int(c.status.item()) == 4 and int(c.free_top.item()) == 1
    lens = sorted(c.seq_len[0].tolist())
    assert lens == [64, 64 + T]
    b = c.seq_len[0].tolist().index(64)
    assert torch.all(out[b] == 7.0) and not torch.any(out[1 - b] == 7.0)
    assert torch.equal(c.K[0, b, :, :64], K[b])


def test_external_scores(B):
    c = Case(B, "dense", 8, 2, 64, [30, 0], [9, 4], external=True).fill(False)
    s = torch.rand((2, c.T, 2), generator=c.gen).to(DEV)
    B.dynts_chunk_step(c.cache.ctx, 0, c.q.to(DEV), c.k_new, c.v_new, c.out, c.scratch, n_new=c.n, s_new=s)
    c.check("external")
    for b, (a, m) in enumerate(zip(c.n_old, c.n_new)):
        assert torch.equal(c.cache.S[0, b, :, a:a + m], s[b, :m].t())
        assert torch.all(c.cache.S[0, b, :, :a] == 0)


def test_lengths_past_the_cache_are_clamped(B):
    """More queries than slots, negative counts."""
    c = Case(B, "dense", 8, 2, 64, [0, 5, 5], [3, 3, 3]).fill(True)
    q = _rand(c.gen, 3, 12, 8, 64)
    out = torch.full((3, 12, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    scratch = torch.empty(B.dynts_chunk_scratch_bytes(c.cache.cfg, 12), dtype=torch.uint8, device=DEV)
    B.dynts_chunk_attend(c.cache.ctx, 0, q.to(DEV), out, scratch, n_new=torch.tensor([100, -3, 8], dtype=torch.int32, device=DEV))
    assert torch.all(out[1] == 7.0)
    for b, m in ((0, 3), (2, 8)):
        assert torch.all(out[b, m:] == 7.0)
        r = plain.attention(q[b], c.K[b], c.V[b], c.pos[b], m, m, 0.125)
        plain.check(out[b, :m], r["out"], r["out_tol"], "clamped")


@pytest.mark.parametrize("layout", ["dense", "paged"])
@pytest.mark.parametrize("T,shape", [(3, {}), (300, {}), (300, dict(window=500))])
def test_a_cache_past_32_bits(B, layout, T, shape):
    """The last head of 1.1 million slots times 32 heads: its elements begin past 2^32.  A chunk's step there against the definition; the
    other sequence is left alone."""
    Hkv, d, n = 16, 128, 1100000
    gen = torch.Generator(device=DEV).manual_seed(9)
    c = (B.Cache if layout == "dense" else B.PagedCache)(1, 2, Hkv, Hkv, d, n + T, 0, 0, 1)
    if layout == "paged":  # the second sequence in the pool's last pages, a head's side by side, the chunk's on the free stack
        page = c.n_pages - Hkv * c.max_pages + torch.arange(Hkv * c.max_pages, dtype=torch.int32, device=DEV).view(Hkv, c.max_pages)
        have = (n + 63) // 64
        c.block_table[0, 1, :, :have] = page[:, :have]
        top = Hkv * (c.max_pages - have)
        c.free_stack[:top] = page[:, have:].reshape(-1).flip(0)
        c.free_top.fill_(top)
    pool_K, pool_V = (c.K, c.V) if layout == "dense" else (c.K_pool, c.V_pool)
    assert pool_K.numel() > 2 ** 32
    rand = lambda *s: torch.randn(s, generator=gen, device=DEV).to(torch.bfloat16)
    K, V = rand(n, d), rand(n, d)
    for pool, x in ((pool_K, K), (pool_V, V)):
        if layout == "dense":
            pool[0, 1, -1, :n] = x
        else:
            pool.view(-1, d)[-c.max_pages * 64:][:n] = x
    c.seq_len[0, 1] = n
    c.next_pos[0, 1] = n
    c.pos[0, 1, :, :n] = torch.arange(n, dtype=torch.int32, device=DEV)
    q, k, v = (rand(2, T, Hkv, d) for _ in range(3))
    q = q * 4  # (few keys carry a row's weight: an output that a wrong place would change)
    out = torch.full((2, T, Hkv, d), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros((2, T, Hkv), device=DEV)
    scratch = torch.empty(B.dynts_chunk_scratch_bytes(c.cfg, T), dtype=torch.uint8, device=DEV)
    n_new = torch.tensor([0, T], dtype=torch.int32, device=DEV)
    B.dynts_chunk_step(c.ctx, 0, q, k, v, out, scratch, lse=lse, n_new=n_new, shaping=B.Shaping(**shape) if shape else None)
    assert int(c.status.item()) == 0 and c.seq_len.tolist() == [[0, n + T]]
    assert torch.all(out[0] == 7.0) and torch.all(c.S[0, 0] == 0)
    r = plain.attention(q[1, :, -1:], torch.cat((K, k[1, :, -1]))[None], torch.cat((V, v[1, :, -1]))[None], torch.arange(n + T)[None], n + T, T,
                        1.0 / math.sqrt(d), device=DEV, **shape)
    plain.check(out[1, :, -1:], r["out"], r["out_tol"], "out")
    plain.check(lse[1, :, -1:], r["lse"], r["lse_tol"], "lse")
    plain.check(c.S[0, 1, -1:, :n + T], r["recv"], r["recv_tol"], "received")


@pytest.mark.parametrize("layout", ["dense", "paged"])
def test_captured_steps(B, layout):
    """A rotation and a chunk's step recorded into a graph and replayed, with eager work between the replays: the same as eager."""
    gen = torch.Generator().manual_seed(6)
    Nb, Hq, Hkv, d, T = 2, 28, 4, 128, 5
    mk = lambda: (B.Cache if layout == "dense" else B.PagedCache)(1, Nb, Hq, Hkv, d, 300, 0, 0, 1)
    a, b = mk(), mk()
    q, k, v = (_rand(gen, Nb, T, h, d).to(DEV) for h in (Hq, Hkv, Hkv))
    rot = B.Rotary(d, torch.rand(64, generator=gen).to(DEV))
    positions = torch.zeros((1, Nb, T), dtype=torch.int32, device=DEV)
    scratch = torch.empty(B.dynts_chunk_scratch_bytes(a.cfg, T), dtype=torch.uint8, device=DEV)
    sh = B.Shaping(softcap=20.0, window=50)

    def step(c, qr, kr, out):
        positions.copy_((c.next_pos[0][:, None] + torch.arange(T, device=DEV)).to(torch.int32)[None])
        B.dynts_rotate(rot, q, k, positions, qr, kr)
        B.dynts_chunk_step(c.ctx, 0, qr, kr, v, out, scratch, shaping=sh)

    bufs = {c: (torch.empty_like(q), torch.empty_like(k), torch.zeros_like(q)) for c in ("a", "b")}
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(b, *bufs["b"])
    torch.cuda.synchronize()
    step(a, *bufs["a"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(b, *bufs["b"])
    assert torch.equal(bufs["a"][2], bufs["b"][2])
    for turn in range(6):
        graph.replay()
        step(a, *bufs["a"])
        torch.cuda.synchronize()
        scratch.fill_(turn)
        assert torch.equal(bufs["a"][2], bufs["b"][2]), turn
        assert torch.equal(a.S, b.S) and torch.equal(a.seq_len, b.seq_len)
        n = int(a.seq_len.max().item())
        assert torch.equal(a.K[:, :, :, :n], b.K[:, :, :, :n])


def test_graphs_that_share_scratch_and_streams_that_do_not(B):
    """Two graphs with one scratch, replayed in turn on one stream; two streams at once, each with a scratch of its own."""
    cases = [Case(B, "dense", 8, 1, 128, [2900, 10], [200, 64], seed=1).fill(True), Case(B, "paged", 28, 4, 128, [900, 333], [40, 77], seed=2).fill(True)]
    qs = [c.q.to(DEV) for c in cases]
    want = []
    for c, q in zip(cases, qs):
        B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n)
        want.append((c.out.clone(), c.lse.clone()))
    shared = torch.empty(max(c.scratch.numel() for c in cases), dtype=torch.uint8, device=DEV)
    graphs = []
    for c, q in zip(cases, qs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, shared, lse=c.lse, n_new=c.n)

    def same():
        torch.cuda.synchronize()
        for c, (out, lse) in zip(cases, want):
            assert torch.equal(c.out, out) and torch.equal(c.lse, lse)
            c.out.fill_(7.0)
            c.lse.fill_(7.0)
        torch.cuda.synchronize()

    same()
    for turn in range(4):
        shared.fill_(turn)
        for graph in graphs:
            graph.replay()
        same()
    streams = [torch.cuda.Stream() for _ in cases]
    for turn in range(4):
        for c, q, stream in zip(cases, qs, streams):
            with torch.cuda.stream(stream):
                B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n)
        same()
        for c, q, stream in zip(cases, qs, streams):
            B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n, stream=stream.cuda_stream)
        same()


def test_results_do_not_change_from_run_to_run(B):
    c = Case(B, "dense", 32, 8, 128, [900, 0, 333], [40, 77, 1]).fill(True)
    q = c.q.to(DEV)
    first = None
    for _ in range(4):
        B.dynts_chunk_attend(c.cache.ctx, 0, q, c.out, c.scratch, lse=c.lse, n_new=c.n)
        dst = torch.zeros((3, 8, c.cap), dtype=torch.float32, device=DEV)
        B.dynts_chunk_scores(c.cache.ctx, 0, q, c.lse, dst=dst, accumulate=False, n_new=c.n)
        got = (c.out.clone(), c.lse.clone(), dst)
        first = first or got
        assert all(torch.equal(x, y) for x, y in zip(first, got))


@pytest.mark.parametrize("layout", ["dense", "paged"])
def test_a_request_from_its_prompt_on(B, layout):
    """Everything together, as a serving program uses it, over two layers: a prompt in two chunks with rotary positions, single
    tokens by dynts_decode_step, a trigger, drafted tokens of which some are dropped again by a compaction, a padded chunk with a
    window and capped logits.  After each chunk its outputs are those of the definition on what the cache then holds."""
    gen = torch.Generator().manual_seed(21)
    L, Nb, Hq, Hkv, d = 2, 3, 28, 4, 128
    budget, window, every = 40, 8, 20
    cap = 200
    c = (B.Cache if layout == "dense" else B.PagedCache)(L, Nb, Hq, Hkv, d, cap, budget, window, every)
    rot = B.Rotary(d, (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).to(torch.float32).to(DEV))
    scratch = torch.empty(B.dynts_chunk_scratch_bytes(c.cfg, 64), dtype=torch.uint8, device=DEV)

    def fresh(T, layer):
        q, k, v = (_rand(gen, Nb, T, h, d).to(DEV) for h in (Hq, Hkv, Hkv))
        at = (c.next_pos[layer][:, None] + torch.arange(T, device=DEV)).to(torch.int32)[None].contiguous()
        B.dynts_rotate(rot, q, k, at, q, k)
        return q, k, v

    def chunk(T, layer, n_new=None, question=False, **shape):
        q, k, v = fresh(T, layer)
        n0 = c.seq_len[layer].tolist()
        out = torch.full((Nb, T, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((Nb, T, Hq), 7.0, dtype=torch.float32, device=DEV)
        n = torch.tensor(n_new, dtype=torch.int32, device=DEV) if n_new else None
        B.dynts_chunk_step(c.ctx, layer, q, k, v, out, scratch, lse=lse, n_new=n, question=question, shaping=B.Shaping(**shape) if shape else None)
        K, V, pos = c.K[layer].cpu(), c.V[layer].cpu(), c.pos[layer].cpu()
        for b in range(Nb):
            m = n_new[b] if n_new else T
            end = n0[b] + m
            assert int(c.seq_len[layer, b]) == end and torch.all(out[b, m:] == 7.0) and torch.all(lse[b, m:] == 7.0)
            assert torch.equal(K[b, :, n0[b]:end], k[b, :m].transpose(0, 1).cpu()) and torch.equal(V[b, :, n0[b]:end], v[b, :m].transpose(0, 1).cpu())
            if m:
                r = plain.attention(q[b].cpu(), K[b], V[b], pos[b], end, m, 1.0 / math.sqrt(d), **shape)
                plain.check(out[b, :m], r["out"], r["out_tol"], "request out")
                plain.check(lse[b, :m], r["lse"], r["lse_tol"], "request lse")

    o = torch.zeros((Nb, Hq, d), dtype=torch.float32, device=DEV)
    for layer in range(L):
        chunk(33, layer, question=True)
        chunk(12, layer, n_new=[12, 5, 0], question=True)
    for _ in range(budget + window + every):
        for layer in range(L):
            q, k, v = (x[:, 0].contiguous() for x in fresh(1, layer))
            B.dynts_decode_step(c.ctx, layer, q, k, v, o)
    for layer in range(L):
        B.dynts_select_evict(c.ctx, layer, c.keep_idx, c.new_len)
        B.dynts_compact(c.ctx, layer, c.keep_idx, c.new_len)
        chunk(6, layer)                                     # drafted
        kept = (c.seq_len[layer] - 4).to(torch.int32)       # four of them are not accepted
        c.keep_idx.copy_(torch.arange(cap, device=DEV, dtype=torch.int32).expand_as(c.keep_idx))
        B.dynts_compact(c.ctx, layer, c.keep_idx, kept)
        c.next_pos[layer] -= 4
        chunk(17, layer, n_new=[0, 17, 9], window=30, softcap=8.0)
        q, k, v = (x[:, 0].contiguous() for x in fresh(1, layer))
        B.dynts_decode_step(c.ctx, layer, q, k, v, o)
        B.dynts_update_scores(c.ctx, layer)
        assert torch.isfinite(o).all()
    assert int(c.status.item()) == 0
    if layout == "paged":
        used, taken = c.pages_in_use()
        assert used == taken
