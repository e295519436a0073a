"""Caches of 8-bit codes (dynts_bind_codes) against the definition in float64."""
import math

import pytest
import torch

from tests import chunk_plain as plain
from tests import codes_plain as held

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
CODES = [1, 2]  # DYNTS_CODE_E4M3, DYNTS_CODE_INT8
LAYOUTS = ["dense", "paged"]


@pytest.fixture(scope="module")
def B():
    from paper_2601_18383_amd import binding
    return binding


def _rand(gen, *shape, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(torch.bfloat16)


def _cache(B, layout, code, Nb, Hq, Hkv, d, cap, budget=0, window=0, every=1, L=1, **kw):
    return B.CodedCache(L, Nb, Hq, Hkv, d, cap, budget, window, every, code=code, paged=layout == "paged", **kw)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _scratch(B, c, T):
    s = torch.empty(B.dynts_codes_scratch_bytes(c.cfg, T), dtype=torch.uint8, device=DEV)
    s.fill_(0xA5)
    return s


def _same(got, ref):
    """Equal, NaN in the same places."""
    got, ref = got.double().cpu(), ref.double()
    return torch.equal(got.isnan(), ref.isnan()) and torch.equal(torch.nan_to_num(got, 0, 0, 0), torch.nan_to_num(ref, 0, 0, 0))


# ---- writing and reading back --------------------------------------------------------------------------------------------

def _special(gen, *shape):
    """Rows with everything that rounding meets: ties, tops of the range, powers of two, tiny and huge blocks, zeros, non-finite blocks."""
    x = _rand(gen, *shape)
    flat = x.view(-1, 32)
    n = flat.shape[0]
    k = torch.arange(n)
    flat *= torch.exp2((k * 7 % 200 - 100).float())[:, None].to(torch.bfloat16)
    ties = torch.arange(32).float() / 2 + 0.5
    for i, top in enumerate((127.0, 127.5, 128.0, 126.5, 448.0, 450.0, 446.0, 480.0, 1.0, 255.0)):
        flat[3 * i] = ties.to(torch.bfloat16)
        flat[3 * i, 5] = top
        flat[3 * i, 6] = -top / 2
    # every step of e4m3 and the points half way, in a block whose scale is 1
    grid = torch.tensor([m * 2.0 ** e for e in range(-10, 8) for m in (8, 8.5, 9, 11.5, 15, 15.5)] + [0.0] * 20)[:96].view(3, 32)
    flat[40:43] = grid.to(torch.bfloat16)
    flat[40:43, 0] = 448.0
    flat[50] = 0
    flat[51] = -0.0
    flat[52] = 2.0 ** -120
    flat[53] = 2.0 ** -133
    flat[54] = 1.99 * 2.0 ** 125
    flat[55, 7] = 2.0 ** 126
    flat[56, 3] = math.inf
    flat[57, 31] = -math.inf
    flat[58, 0] = math.nan
    flat[59] = 3.38e38
    return x


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("d", [64, 128])
def test_rounding(B, layout, code, d):
    gen = torch.Generator().manual_seed(d + code)
    Nb, Hkv, T = 2, 2, 50
    k, v = _special(gen, Nb, T, Hkv, d), _special(gen, Nb, T, Hkv, d).flip(1)
    c = _cache(B, layout, code, Nb, 4, Hkv, d, 70)
    B.dynts_chunk_append(c.ctx, 0, k.to(DEV), v.to(DEV), _scratch(B, c, T))
    ko, vo = torch.full((Nb, Hkv, T, d), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((Nb, Hkv, T, d), 7.0, dtype=torch.bfloat16, device=DEV)
    B.dynts_read_rows(c.ctx, 0, ko, vo)
    assert _same(ko, held.hold(k, code).transpose(1, 2)) and _same(vo, held.hold(v, code).transpose(1, 2))
    # what is read back, written again, is the same (but for a block whose largest was rounded up to 2^126, which is no longer one that is held)
    again = _cache(B, layout, code, Nb, 4, Hkv, d, 70)
    B.dynts_chunk_append(again.ctx, 0, ko.transpose(1, 2).contiguous(), vo.transpose(1, 2).contiguous(), _scratch(B, c, T))
    for got, once in ((again.K[0][:, :, :T], ko.cpu()), (again.V[0][:, :, :T], vo.cpu())):
        large = (once.float().unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True) >= 2.0 ** 126).expand(*once.shape[:-1], -1, 32).flatten(-2)
        assert _same(got, torch.where(large, math.nan, once.double())) and _same(got, held.hold(once, code))
        assert int(large.sum()) <= 3 * 32


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("Hkv,d,turns", [(2, 64, [[1, 0, 3], [65, 1, 0], [200, 64, 63]]), (8, 128, [[0, 1, 1], [1, 1, 1], [513, 300, 77]]),
                                         (4, 128, [[32, 0, 31], [32, 33, 1]])])
def test_append_in_turns(B, layout, code, Hkv, d, turns):
    """Chunks of several lengths one after the other, small (one launch) and large; padding holds NaN; scores and positions as in a bf16 cache."""
    gen = torch.Generator().manual_seed(5)
    Nb, total = 3, [sum(t[b] for t in turns) for b in range(3)]
    cap = max(total) + 3
    c = _cache(B, layout, code, Nb, Hkv, Hkv, d, cap)
    K, V = _rand(gen, Nb, Hkv, cap, d), _rand(gen, Nb, Hkv, cap, d, scale=30.0)
    done = [0] * Nb
    for i, t in enumerate(turns):
        T = max(t) + 2
        rows = lambda x: torch.stack([torch.cat((x[b, :, done[b]:done[b] + m].transpose(0, 1), torch.full((T - m, Hkv, d), math.nan, dtype=x.dtype)))
                                      for b, m in enumerate(t)]).contiguous().to(DEV)
        B.dynts_chunk_append(c.ctx, 0, rows(K), rows(V), _scratch(B, c, T), n_new=_ints(t), question=i == 0)
        done = [a + m for a, m in zip(done, t)]
    assert c.seq_len[0].tolist() == done and c.next_pos[0].tolist() == done and c.n_prompt.tolist() == turns[0]
    got_k, got_v = c.K[0], c.V[0]
    for b, n in enumerate(done):
        assert _same(got_k[b, :, :n], held.hold(K[b, :, :n], code)) and _same(got_v[b, :, :n], held.hold(V[b, :, :n], code))
        assert torch.all(got_k[b, :, n:] == 0)
        assert torch.equal(c.pos[0, b, :, :n].cpu(), torch.arange(n, dtype=torch.int32).expand(Hkv, n))
        assert torch.all(torch.isinf(c.S[0, b, :, :turns[0][b]])) and torch.all(c.S[0, b, :, turns[0][b]:n] == 0)
    assert int(c.status.item()) == 0
    if layout == "paged":
        assert len(set(c.pages_in_use())) == 1


@pytest.mark.parametrize("kind", ["dense", "paged", "e4m3", "int8_paged"])
def test_read_rows_of_any_cache(B, kind):
    """From another slot in every sequence; slots that a sequence does not have leave their rows as they were."""
    gen = torch.Generator().manual_seed(3)
    Nb, Hkv, d, cap, lens = 4, 2, 64, 150, [150, 70, 1, 0]
    k, v = _rand(gen, Nb, cap, Hkv, d), _rand(gen, Nb, cap, Hkv, d)
    if kind in LAYOUTS:
        c = (B.Cache if kind == "dense" else B.PagedCache)(2, Nb, 4, Hkv, d, cap, 0, 0, 1)
        values = (k.double(), v.double())
    else:
        code = 1 if kind == "e4m3" else 2
        c = _cache(B, "paged" if "paged" in kind else "dense", code, Nb, 4, Hkv, d, cap, L=2)
        values = (held.hold(k, code), held.hold(v, code))
    scratch = torch.empty(B.dynts_codes_scratch_bytes(c.cfg, cap), dtype=torch.uint8, device=DEV)
    for layer in (1, 0):
        B.dynts_chunk_append(c.ctx, layer, k.to(DEV) * (1 + layer), v.to(DEV), scratch, n_new=_ints(lens))
    for layer in (0, 1):
        for first, n_rows in (([0, 0, 0, 0], 150), ([100, 69, 0, 0], 60), ([149, 70, 1, 5], 1), ([-3, 2 ** 31 - 1, -2 ** 31, 0], 10), (None, 7)):
            ko = torch.full((Nb, Hkv, n_rows, d), 7.0, dtype=torch.bfloat16, device=DEV)
            vo = ko.clone()
            B.dynts_read_rows(c.ctx, layer, ko, vo, first=_ints(first) if first else None)
            for b in range(Nb):
                for i in range(n_rows):
                    j = (first[b] if first else 0) + i
                    want = [x[b, j] * f if 0 <= j < lens[b] else torch.full((Hkv, d), 7.0).double() for x, f in zip(values, (1 + layer, 1))]
                    assert torch.equal(ko[b, :, i].double().cpu(), want[0]) and torch.equal(vo[b, :, i].double().cpu(), want[1])


# ---- attention and scores ---------------------------------------------------------------------------------------------------

class Case:
    """A cache of codes with n_old slots before n_new tokens, all of them appended."""

    def __init__(self, B, layout, code, Hq, Hkv, d, n_old, n_new, gaps=0, seed=0, qscale=1.5, T=None, external=False):
        gen = self.gen = torch.Generator().manual_seed(seed + d + Hq)
        self.B, self.n_old, self.n_new, self.Hq, self.Hkv, self.d = B, n_old, n_new, Hq, Hkv, d
        Nb, self.T = len(n_old), T or max(max(n_new), 1)
        self.cap = max(a + m for a, m in zip(n_old, n_new)) + 5
        K, V = _rand(gen, Nb, self.cap, Hkv, d), _rand(gen, Nb, self.cap, Hkv, d)
        self.q = _rand(gen, Nb, self.T, Hq, d, scale=qscale)
        self.c = c = _cache(B, layout, code, Nb, Hq, Hkv, d, self.cap, external_scores=external)
        total = [a + m for a, m in zip(n_old, n_new)]
        s = torch.zeros((Nb, self.cap, Hkv), dtype=torch.float32, device=DEV) if external else None
        B.dynts_chunk_append(c.ctx, 0, K.to(DEV), V.to(DEV), _scratch(B, c, self.cap), n_new=_ints(total), s_new=s)
        self.K, self.V = held.hold(K, code).transpose(1, 2), held.hold(V, code).transpose(1, 2)
        self.pos = []
        for b, (a, m) in enumerate(zip(n_old, n_new)):
            extra = torch.floor(torch.rand((Hkv, a), generator=gen).sort(dim=-1).values * (gaps + 1))
            p = torch.cat((torch.arange(a) + extra, (a + gaps + torch.arange(m)).expand(Hkv, m)), dim=1).to(torch.int32)
            self.pos.append(p)
            c.pos[0, b, :, :a + m] = p.to(DEV)
            c.next_pos[0, b] = a + gaps + m
        self.scratch = _scratch(B, c, self.T)
        for b, m in enumerate(n_new):
            self.q[b, m:] = math.nan
        self.out = torch.full((Nb, self.T, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((Nb, self.T, Hq), 7.0, dtype=torch.float32, device=DEV)
        self.dst = torch.full((Nb, Hkv, self.cap), 7.0, dtype=torch.float32, device=DEV)

    def run(self, shaping=None):
        B, c, q, n = self.B, self.c, self.q.to(DEV), _ints(self.n_new)
        B.dynts_chunk_attend(c.ctx, 0, q, self.out, self.scratch, lse=self.lse, n_new=n, shaping=shaping)
        B.dynts_chunk_scores(c.ctx, 0, q, self.lse, dst=self.dst, accumulate=False, n_new=n, shaping=shaping)
        return self

    def check(self, **shape):
        per = {k: shape.pop(k, None) for k in ("first", "last")}
        worst = {}
        for b, (a, m) in enumerate(zip(self.n_old, self.n_new)):
            assert torch.all(self.out[b, m:] == 7.0) and torch.all(self.lse[b, m:] == 7.0)
            assert torch.all(self.dst[b, :, (a + m if m else 0):] == 7.0)
            if m == 0:
                continue
            r = plain.attention(self.q[b], self.K[b], self.V[b], self.pos[b], a + m, m, 1.0 / math.sqrt(self.d), **shape,
                                **{k: (v[b] if v is not None else None) for k, v in per.items()})
            for name, got in (("out", self.out[b, :m]), ("lse", self.lse[b, :m]), ("recv", self.dst[b, :, :a + m])):
                worst[name] = max(worst.get(name, 0.0), plain.check(got, r[name], r[name + "_tol"], "%s[%d]" % (name, b)))
        assert int(self.c.status.item()) == 0
        print(worst)


SHAPES = [  # Hq, Hkv, d, n_old, n_new
    (8, 2, 64, [0, 1, 63, 64, 200, 129, 31], [1, 1, 1, 1, 1, 1, 0]),    # single tokens, lengths around tiles and pages
    (28, 4, 128, [0, 31, 32, 300, 64], [1, 1, 1, 1, 1]),
    (28, 4, 128, [0, 5, 300, 64], [37, 0, 12, 64]),                     # odd groups, an empty chunk, an empty cache
    (6, 6, 128, [130, 77], [33, 65]),                                   # no sharing of KV heads
    (16, 1, 64, [500, 3], [9, 100]),                                    # the largest group
    (16, 1, 128, [40], [257]),
    (8, 1, 128, [3000, 10], [20, 4]),                                   # keys in shares; a short cache beside it
    (8, 1, 64, [4000, 900], [2, 1]),
    (28, 4, 128, [0, 31, 32, 33, 100, 257, 64, 1, 5, 0, 90, 128], [60, 60, 1, 59, 0, 33, 60, 37, 32, 31, 64, 7]),  # many rows of many units
    (16, 8, 64, [0, 1, 63, 64, 65, 200, 31, 0] * 2, [150, 149, 64, 1, 0, 128, 65, 150] * 2),
    (8, 2, 128, [8000], [600]),                                         # many rows of few units: keys in shares
]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", SHAPES)
def test_attend_and_scores(B, layout, code, Hq, Hkv, d, n_old, n_new):
    Case(B, layout, code, Hq, Hkv, d, n_old, n_new, gaps=50).run().check()


MANY = [  # as many units as it takes for workgroups of 64 and of 128 rows, in groups of waves and not, and for codes that are unpacked beforehand
    (16, 8, 128, [0, 1, 31, 32, 33, 63, 64, 65, 96, 97] * 2, [30, 30, 1, 29, 0, 17, 32, 30, 16, 30] * 2),
    (28, 4, 128, [0, 300, 64, 95] * 4, [30, 30, 11, 0] * 4),
    (16, 8, 64, [2100, 0, 1, 130] * 4, [64, 64, 33, 5] * 4),
    (16, 8, 64, [0, 33, 64, 190] * 2, [150, 149, 64, 1] * 2),
    (20, 10, 128, [0, 31, 64, 129] * 4, [130, 64, 129, 3] * 4),
    (16, 4, 64, [90, 0, 1, 33], [700, 650, 1, 129]),
]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", MANY)
def test_many_rows_of_many_units(B, layout, code, Hq, Hkv, d, n_old, n_new):
    Case(B, layout, code, Hq, Hkv, d, n_old, n_new, gaps=20, seed=5).run().check()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", [(8, 1, 128, [2100, 10, 700], [2, 1, 0]), (8, 2, 64, [1700, 3], [1, 1]), (8, 1, 128, [2100, 10], [20, 4]),
                                                  (8, 1, 64, [1, 1600], [3, 9]), (16, 1, 128, [1600, 50, 0, 1], [131, 130, 131, 1])])
def test_two_to_four_shares(B, layout, code, Hq, Hkv, d, n_old, n_new):
    Case(B, layout, code, Hq, Hkv, d, n_old, n_new, gaps=20, seed=6).run().check()


def _shapings(c, kind):
    Nb = len(c.n_old)
    own = torch.stack([c.pos[b][0, c.n_old[b]:][:1].expand(1) if c.n_new[b] else torch.zeros(1, dtype=torch.int32) for b in range(Nb)]) + torch.arange(c.T)
    own = own.to(torch.int32)
    s = {}
    if "cap" in kind:
        s["softcap"] = 200.0 if "far" in kind else 3.0
    if "slope" in kind:
        s["slope"] = (2.0 ** (-8.0 * (1 + torch.arange(c.Hq)) / c.Hq)).to(torch.float32)
    if "window" in kind:
        s["window"] = 40
    if "documents" in kind:
        s["first"] = (own // 23 * 23).to(torch.int32)
    if "empty" in kind:  # rows that see nothing
        first, last = torch.zeros_like(own), own.clone()
        first[:, ::3], last[:, ::3] = 10, 9
        s["first"], s["last"] = first, last
    return s


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("kind", ["cap", "cap_far_window", "slope", "window", "documents", "empty", "cap_slope_window_empty"])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", [SHAPES[0], SHAPES[1], SHAPES[2], SHAPES[6], SHAPES[8], SHAPES[9]])
def test_shaped(B, layout, code, kind, Hq, Hkv, d, n_old, n_new):
    c = Case(B, layout, code, Hq, Hkv, d, n_old, n_new, gaps=90, seed=11)
    s = _shapings(c, kind)
    c.run(B.Shaping(**{k: (v.to(DEV) if torch.is_tensor(v) else v) for k, v in s.items()})).check(**s)


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("many", [False, True])
def test_hidden_keys_may_be_anything(B, code, many):
    """Blocks without a scale in rows of K that nobody sees, and whatever lies behind the length."""
    c = Case(B, "dense", code, 8, 2, 64, [100], [700 if many else 7], seed=3)
    c.c.K_scale[0, :, :, :50] = 255
    n = 100 + c.n_new[0]
    for t in (c.c.K_codes, c.c.V_codes, c.c.K_scale, c.c.V_scale):
        t[0, :, :, n:] = 255
    first = torch.full((1, c.T), 50, dtype=torch.int32)
    c.K[:, :, :50] = 0
    c.run(B.Shaping(first=first.to(DEV))).check(first=first)


@pytest.mark.parametrize("code", CODES)
def test_a_seen_row_without_a_scale_shows(B, code):
    """A NaN that is written comes back as NaN in the outputs of the tokens that see it, and only there."""
    gen = torch.Generator().manual_seed(1)
    c = _cache(B, "dense", code, 1, 4, 2, 64, 100)
    k, v = _rand(gen, 1, 60, 2, 64), _rand(gen, 1, 60, 2, 64)
    v[0, 30, 1, 5] = math.nan
    out = torch.zeros((1, 60, 4, 64), dtype=torch.bfloat16, device=DEV)
    B.dynts_chunk_step(c.ctx, 0, _rand(gen, 1, 60, 4, 64).to(DEV), k.to(DEV), v.to(DEV), out, _scratch(B, c, 60))
    nan = out.isnan().cpu()
    assert torch.all(nan[0, 30:, 2:, :32]) and not nan[0, :, :2].any() and not nan[0, :, 2:, 32:].any()


def test_far_rows(B):
    """Codes and scales past 2^32 bytes: the last units of a large cache."""
    Nb, Hkv, d, cap = 5, 8, 128, 1 << 20
    c = _cache(B, "dense", 2, Nb, Hkv, Hkv, d, cap)
    assert c.K_codes.numel() > 1 << 32
    gen = torch.Generator().manual_seed(2)
    n = [0, 0, 0, 0, 70]
    k, v = _rand(gen, Nb, 70, Hkv, d), _rand(gen, Nb, 70, Hkv, d)
    c.seq_len[0, 4] = c.next_pos[0, 4] = cap - 70
    c.pos[0, 4] = torch.arange(cap, dtype=torch.int32, device=DEV)
    scratch = torch.empty(B.dynts_chunk_scratch_bytes(c.cfg, 70), dtype=torch.uint8, device=DEV)
    scratch = torch.empty(max(scratch.numel(), B.dynts_codes_scratch_bytes(c.cfg, 70)), dtype=torch.uint8, device=DEV)
    B.dynts_chunk_append(c.ctx, 0, k.to(DEV), v.to(DEV), scratch, n_new=_ints(n))
    ko = torch.zeros((Nb, Hkv, 70, d), dtype=torch.bfloat16, device=DEV)
    vo = torch.zeros_like(ko)
    B.dynts_read_rows(c.ctx, 0, ko, vo, first=_ints([cap - 70] * Nb))
    assert _same(ko[4], held.hold(k[4], 2).transpose(0, 1)) and _same(vo[4], held.hold(v[4], 2).transpose(0, 1)) and not ko[:4].any()
    # the last two tokens attend to a window at the far end
    q = _rand(gen, Nb, 2, Hkv, d)
    out, lse = torch.zeros((Nb, 2, Hkv, d), dtype=torch.bfloat16, device=DEV), torch.zeros((Nb, 2, Hkv), dtype=torch.float32, device=DEV)
    B.dynts_chunk_attend(c.ctx, 0, q.to(DEV), out, scratch, lse=lse, n_new=_ints([0, 0, 0, 0, 2]), shaping=B.Shaping(window=60))
    Kv, Vv = held.hold(k[4], 2).transpose(0, 1), held.hold(v[4], 2).transpose(0, 1)
    r = plain.attention(q[4], Kv, Vv, torch.arange(70).expand(Hkv, 70), 70, 2, 1 / math.sqrt(d), window=60)
    plain.check(out[4], r["out"], r["out_tol"], "out")
    plain.check(lse[4], r["lse"], r["lse_tol"], "lse")


# ---- the whole decode ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("Hq,Hkv,d,external", [(8, 2, 64, False), (28, 4, 128, False), (4, 4, 128, True)])
def test_decode_with_triggers(B, layout, code, Hq, Hkv, d, external):
    """A request from its prompt on, in single tokens and chunks, with evictions, beside a bf16 cache that is given the values that the codes stand
    for: the same lengths and positions, rows bit for bit, scores and outputs within the difference of their sums' order."""
    gen = torch.Generator().manual_seed(8)
    Nb, budget, window, every = 3, 40, 12, 30
    prompt = [10, 4, 70]
    cap = max(prompt) + budget + window + every + 30
    kw = dict(external_scores=external)
    a = _cache(B, layout, code, Nb, Hq, Hkv, d, cap, budget, window, every, **kw)
    b = (B.Cache if layout == "dense" else B.PagedCache)(1, Nb, Hq, Hkv, d, cap, budget, window, every, **kw)
    scratch = _scratch(B, a, 80)
    trig = torch.zeros((Nb,), dtype=torch.uint8, device=DEV)
    evictions = 0
    for turn, T in enumerate([70, 1, 1, 24, 7, 1, 16, 30, 5, 24, 1, 1, 30, 2]):
        q = _rand(gen, Nb, T, Hq, d, scale=2.0).to(DEV)
        k, v = _rand(gen, Nb, T, Hkv, d), _rand(gen, Nb, T, Hkv, d)
        n = prompt if turn == 0 else [T, T, max(0, T - 1)] if turn % 2 else [T] * Nb
        s = torch.rand((Nb, T, Hkv), generator=gen).to(DEV) if external else None
        outs = []
        for c, kk, vv in ((a, k, v), (b, held.hold(k, code).to(torch.bfloat16), held.hold(v, code).to(torch.bfloat16))):
            out, lse = torch.zeros((Nb, T, Hq, d), dtype=torch.bfloat16, device=DEV), torch.zeros((Nb, T, Hq), dtype=torch.float32, device=DEV)
            B.dynts_chunk_step(c.ctx, 0, q, kk.to(DEV), vv.to(DEV), out, scratch, lse=lse, n_new=_ints(n), s_new=s, question=turn == 0)
            outs.append((out.double(), lse.double()))
        # (either rounds weights and outputs: 2^-7 of what is summed, values of size 6 at most, twice over)
        assert (outs[0][0] - outs[1][0]).abs().max() <= 2 * 6 * 2.0 ** -7 and (outs[0][1] - outs[1][1]).abs().max() <= 1e-4
        assert (a.S - b.S)[torch.isfinite(b.S)].abs().max() <= 1e-3 and torch.equal(torch.isinf(a.S), torch.isinf(b.S))
        b.S.copy_(a.S)  # (so that near ties fall the same way)
        due = (a.seq_len[0] - a.n_prompt) >= budget + window
        trig.copy_(due.to(torch.uint8))
        if bool(due.any()):
            evictions += 1
            for c in (a, b):
                B.dynts_select_evict(c.ctx, 0, c.keep_idx, c.new_len, trigger=trig)
            assert torch.equal(a.new_len, b.new_len)
            for c in (a, b):
                B.dynts_compact(c.ctx, 0, c.keep_idx, c.new_len, trigger=trig)
        assert torch.equal(a.seq_len, b.seq_len) and torch.equal(a.next_pos, b.next_pos) and torch.equal(a.n_prompt, b.n_prompt)
        ak, av, bk, bv = a.K[0], a.V[0], b.K[0], b.V[0]
        for i, m in enumerate(a.seq_len[0].tolist()):
            assert torch.equal(ak[i, :, :m], bk[i, :, :m]) and torch.equal(av[i, :, :m], bv[i, :, :m])
            assert torch.equal(a.pos[0, i, :, :m], b.pos[0, i, :, :m]) and torch.equal(a.S[0, i, :, :m], b.S[0, i, :, :m])
    assert evictions >= 4 and int(a.status.item()) == 0
    if layout == "paged":
        assert len(set(a.pages_in_use())) == 1


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
def test_compact_large(B, layout, d):
    """Thousands of rows, scattered keeps, none moved, all dropped, sequences without a trigger."""
    gen = torch.Generator().manual_seed(4)
    Nb, Hkv, cap = 4, 2, 5000
    lens = [5000, 4097, 300, 129]
    c = _cache(B, layout, 2, Nb, Hkv, Hkv, d, cap, L=2)
    k, v = _rand(gen, Nb, cap, Hkv, d), _rand(gen, Nb, cap, Hkv, d)
    scratch = torch.empty(B.dynts_codes_scratch_bytes(c.cfg, cap), dtype=torch.uint8, device=DEV)
    for layer in (0, 1):
        B.dynts_chunk_append(c.ctx, layer, k.to(DEV), v.to(DEV), scratch, n_new=_ints(lens))
    c.S[1] = torch.rand(c.S[1].shape, generator=gen).to(DEV)
    before = [t.clone() for t in (c.K[1], c.V[1], c.S[1], c.pos[1])]
    other = c.K[0].clone()
    new = [2500, 4000, 300, 0]
    keep = torch.zeros((Nb, Hkv, cap), dtype=torch.int32)
    for b in range(Nb):
        for h in range(Hkv):
            keep[b, h, :new[b]] = torch.randperm(lens[b], generator=gen)[:new[b]].sort().values.to(torch.int32)
    trigger = torch.tensor([1, 1, 1, 1], dtype=torch.uint8, device=DEV)
    trigger[2] = 0
    B.dynts_compact(c.ctx, 1, keep.to(DEV), _ints(new), trigger=trigger)
    assert c.seq_len[1].tolist() == [2500, 4000, 300, 0] and c.seq_len[0].tolist() == lens
    after = [c.K[1], c.V[1], c.S[1], c.pos[1]]
    for b in (0, 1):
        for h in range(Hkv):
            at = keep[b, h, :new[b]].long().to(DEV)
            for x, y in zip(before, after):
                assert torch.equal(x[b, h][at], y[b, h, :new[b]])
    assert torch.equal(before[0][2, :, :300], after[0][2, :, :300]) and torch.equal(other, c.K[0])
    if layout == "paged":
        assert len(set(c.pages_in_use())) == 1


@pytest.mark.parametrize("layout", LAYOUTS)
def test_chunks_that_do_not_fit(B, layout):
    """Full caches and a dry pool leave their sequences alone."""
    gen = torch.Generator().manual_seed(6)
    Nb, Hkv, d, cap = 3, 2, 128, 100
    kw = dict(n_pages=2 * 2 * Nb - 2) if layout == "paged" else {}
    c = _cache(B, layout, 1, Nb, 4, Hkv, d, cap, **kw)
    scratch = _scratch(B, c, 70)
    k, v = _rand(gen, Nb, 70, Hkv, d).to(DEV), _rand(gen, Nb, 70, Hkv, d).to(DEV)
    B.dynts_chunk_append(c.ctx, 0, k, v, scratch, n_new=_ints([60, 60, 40]))
    assert int(c.status.item()) == 0
    rows = c.K.clone()
    B.dynts_chunk_append(c.ctx, 0, k, v, scratch, n_new=_ints([41, 30, 0]))
    assert int(c.status.item()) == 1 and c.seq_len[0].tolist() == [60, 90, 40]
    assert torch.equal(c.K[0, 0], rows[0, 0]) and torch.equal(c.K[0, 2], rows[0, 2])
    if layout == "paged":  # two pages a head for sequence 1: two of ten are left, and sequences 0 and 2 ask for two each
        B.dynts_chunk_append(c.ctx, 0, k, v, scratch, n_new=_ints([20, 0, 30]))
        assert int(c.status.item()) == 5 and sorted(c.seq_len[0].tolist()) in ([40, 80, 90], [60, 70, 90])
        assert len(set(c.pages_in_use())) == 1


@pytest.mark.parametrize("T", [1, 100])
def test_recorded_steps(B, T):
    """A chunk's step recorded and replayed, with eager work between the replays: as eager steps on a cache beside it."""
    gen = torch.Generator().manual_seed(7)
    Nb, Hq, Hkv, d, cap = 12, 28, 4, 128, 700
    one, two = (_cache(B, "paged", 2, Nb, Hq, Hkv, d, cap) for _ in range(2))
    scratch = _scratch(B, one, 100)
    q, k, v = (torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in ((Nb, T, Hq, d), (Nb, T, Hkv, d), (Nb, T, Hkv, d)))
    out, ref = torch.zeros_like(q), torch.zeros_like(q)
    B.dynts_chunk_step(one.ctx, 0, q, k, v, out, scratch)
    B.dynts_chunk_step(two.ctx, 0, q, k, v, ref, scratch)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        B.dynts_chunk_step(one.ctx, 0, q, k, v, out, scratch)
    for _ in range(4):
        q.copy_(_rand(gen, Nb, T, Hq, d))
        k.copy_(_rand(gen, Nb, T, Hkv, d))
        v.copy_(_rand(gen, Nb, T, Hkv, d))
        graph.replay()
        torch.cuda.synchronize()
        B.dynts_chunk_step(two.ctx, 0, q, k, v, ref, scratch)
        assert torch.equal(out, ref) and torch.equal(one.S, two.S) and torch.equal(one.seq_len, two.seq_len)
        torch.cuda.synchronize()
    assert torch.equal(one.K, two.K) and torch.equal(one.V, two.V)


def test_two_streams(B):
    """Two caches on two streams at once, each with scratch of its own, against one after the other."""
    gen = torch.Generator().manual_seed(9)
    Nb, Hq, Hkv, d, T = 16, 28, 4, 128, 60
    data = [(_rand(gen, Nb, T, Hq, d).to(DEV), _rand(gen, Nb, T, Hkv, d).to(DEV), _rand(gen, Nb, T, Hkv, d).to(DEV)) for _ in range(2)]
    results = []
    for together in (False, True):
        caches = [_cache(B, "dense", 1 + i, Nb, Hq, Hkv, d, 400) for i in range(2)]
        outs = [torch.zeros_like(data[i][0]) for i in range(2)]
        scratch = [_scratch(B, caches[i], T) for i in range(2)]
        streams = [torch.cuda.Stream() if together else torch.cuda.current_stream() for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(5):
            for i in range(2):
                B.dynts_chunk_step(caches[i].ctx, 0, *data[i], outs[i], scratch[i], stream=streams[i])
        torch.cuda.synchronize()
        results.append([t.clone() for i in range(2) for t in (outs[i], caches[i].S, caches[i].K_codes, caches[i].K_scale)])
    assert all(torch.equal(x, y) for x, y in zip(*results))


def test_rows_of_many_heads(B):
    """More rows than 2^25 in one chunk, of a number of heads that is no power of two, on a bf16 cache: every row where it belongs."""
    Hkv, d, T = 127, 64, 330000
    c = B.Cache(1, 1, Hkv, Hkv, d, T + 64, 0, 0, 1)
    gen = torch.Generator(device=DEV).manual_seed(1)
    k = torch.randint(-30000, 30000, (1, T, Hkv, d), generator=gen, device=DEV, dtype=torch.int16).view(torch.bfloat16)
    scratch = torch.empty(B.dynts_chunk_scratch_bytes(c.cfg, T), dtype=torch.uint8, device=DEV)
    B.dynts_chunk_append(c.ctx, 0, k, k, scratch)
    assert int(c.status.item()) == 0 and int(c.seq_len.item()) == T
    for h in list(range(0, Hkv, 9)) + [Hkv - 1]:
        assert torch.equal(c.K[0, 0, h, :T].view(torch.int16), k[0, :, h].view(torch.int16)), h
        assert torch.equal(c.V[0, 0, h, :T].view(torch.int16), k[0, :, h].view(torch.int16)), h
        assert torch.equal(c.pos[0, 0, h, :T], torch.arange(T, dtype=torch.int32, device=DEV))
    assert not c.K[0, 0, :, T:].any()
