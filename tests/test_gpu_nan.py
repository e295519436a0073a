"""A NaN in a row of K: it shows in the outputs, the lse and the received weights of the tokens that see it, whichever kernel they are given to and however many shares
their keys are cut into, and nowhere else."""
import math

import pytest
import torch

from tests import chunk_plain as plain
from tests import codes_plain as held
from tests.test_gpu_tree import DEV, KINDS, Draft, _code

pytestmark = pytest.mark.gpu

SHAPES = [  # Hq, Hkv, d, n_old, n_new
    (8, 2, 64, [70, 5, 33], [1, 3, 2]),                      # few rows, and up to 16 of codes
    (28, 4, 128, [40, 300], [1, 1]),
    (8, 1, 128, [2100, 10], [2, 1]),                         # two to four shares
    (8, 1, 128, [3000, 600], [20, 4]),                       # five
    (8, 1, 64, [4000, 900], [64, 1]),
    (16, 1, 128, [1600, 50], [131, 130]),                    # many rows, in shares
    (8, 2, 128, [8000], [600]),
    (16, 8, 128, [0, 31, 32, 97] * 5, [30, 17, 1, 30] * 5),  # many units: workgroups of 64 rows in groups of waves
    (16, 8, 64, [0, 33, 64, 190] * 2, [150, 149, 64, 1] * 2),
    (20, 10, 128, [0, 31, 64, 129] * 4, [130, 64, 129, 3] * 4),
]


@pytest.fixture(scope="module")
def B():
    from paper_2601_18383_amd import binding
    return binding


def _poison(x, b, h, slot):
    """Element 5 of a row of K, on codes its block, in the cache of a Draft.  In what it is compared with the row is 0: whoever sees it is told by masks."""
    c, at = x.c, (0, b, h, slot)
    if "paged" in x.kind:
        at = (int(c.block_table[0, b, h, slot // 64]), slot % 64)
    if _code(x.kind):
        c.K_codes[at][:32] = 0x7f if _code(x.kind) == 1 else 0
        c.K_scale[at][0] = 255
    else:
        (c.K_pool if x.kind == "paged" else c.K)[at][5] = math.nan
    x.K[b, h, slot] = 0


def _check(got, ref, tol, nan, what):
    """NaN where `nan` says so and nowhere else; the rest within tol."""
    got = got.double().cpu()
    assert torch.equal(got.isnan(), nan.expand(got.shape)), "%s: NaN in %d places instead of %d" % (what, int(got.isnan().sum()), int(nan.expand(got.shape).sum()))
    plain.check(torch.nan_to_num(got, 0.0, math.inf, -math.inf), torch.where(nan.expand(ref.shape), 0.0, ref), torch.where(nan.expand(tol.shape), 0.0, tol), what)


def _places(x):
    """Of every sequence: KV head and slot of a NaN, in the cache, at its very end or in the chunk; None in the last sequence of several."""
    gen = torch.Generator().manual_seed(len(x.n_old) + x.d)
    out = []
    for b, (a, m) in enumerate(zip(x.n_old, x.n_new)):
        slot = [a // 3, a + m - 1, a + m // 2][b % 3]
        out.append(None if b and b == len(x.n_old) - 1 or not a + m else (int(torch.randint(0, x.K.shape[1], (1,), generator=gen)), slot))
    return out


def _attend(x, b, place, **shape):
    """The definition on sequence b: what plain.attention says, and which rows and slots are NaN: [m][Hq], [Hkv][n]."""
    a, m = x.n_old[b], x.n_new[b]
    n, Hkv, G = a + m, x.K.shape[1], x.Hq // x.K.shape[1]
    r = plain.attention(x.q[b], x.K[b], x.V[b], torch.arange(n).expand(Hkv, n), n, m, 1.0 / math.sqrt(x.d), **shape)
    own = a + torch.arange(m)
    seen = torch.arange(n)[None] <= own[:, None]
    if shape.get("window"):
        seen &= torch.arange(n)[None] > own[:, None] - shape["window"]
    rows, slots = torch.zeros((m, x.Hq), dtype=torch.bool), torch.zeros((Hkv, n), dtype=torch.bool)
    if place:
        h, slot = place
        rows[:, h * G:(h + 1) * G] = seen[:, slot][:, None]
        slots[h] = seen[seen[:, slot]].any(0)
    return r, rows, slots


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", SHAPES)
def test_chunks(B, kind, window, Hq, Hkv, d, n_old, n_new):
    x = Draft(B, kind, Hq, Hkv, d, n_old, n_new, seed=31)
    places = _places(x)
    for b, place in enumerate(places):
        if place:
            _poison(x, b, *place)
    shaping = B.Shaping(window=window) if window else None
    dst = torch.zeros((len(n_old), Hkv, x.cap), dtype=torch.float32, device=DEV)
    B.dynts_chunk_attend(x.c.ctx, 0, x.q.to(DEV), x.out, x.scratch, lse=x.lse, n_new=x.n, shaping=shaping)
    B.dynts_chunk_scores(x.c.ctx, 0, x.q.to(DEV), x.lse, dst=dst, accumulate=False, n_new=x.n, shaping=shaping)
    for b, (a, m) in enumerate(zip(n_old, n_new)):
        r, rows, slots = _attend(x, b, places[b], **(dict(window=window) if window else {}))
        _check(x.out[b, :m], r["out"], r["out_tol"], rows[:, :, None], "out[%d]" % b)
        _check(x.lse[b, :m], r["lse"], r["lse_tol"], rows, "lse[%d]" % b)
        _check(dst[b, :, :a + m], r["recv"], r["recv_tol"], slots, "received[%d]" % b)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", SHAPES)
def test_drafts(B, kind, Hq, Hkv, d, n_old, n_new):
    x = Draft(B, kind, Hq, Hkv, d, n_old, n_new, seed=32)
    places = _places(x)
    for b, place in enumerate(places):
        if place:
            _poison(x, b, *place)
    x.attend()
    for b, (a, m) in enumerate(zip(n_old, n_new)):
        r = held.attention(x.q[b], x.K[b], x.V[b], a + m, m, x.masks[b], 1.0 / math.sqrt(d))
        rows = torch.zeros((m, Hq), dtype=torch.bool)
        if places[b]:
            h, slot = places[b]
            G = Hq // Hkv
            rows[:, h * G:(h + 1) * G] = (torch.ones(m, dtype=torch.bool) if slot < a else x.masks[b][:, slot - a])[:, None]
        _check(x.out[b, :m], r["out"], r["out_tol"], rows[:, :, None], "out[%d]" % b)
        _check(x.lse[b, :m], r["lse"], r["lse_tol"], rows, "lse[%d]" % b)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", SHAPES)
def test_whole_steps(B, kind, Hq, Hkv, d, n_old, n_new):
    """A NaN among the rows that a step appends itself; the weights go to the cache's own scores."""
    x = Draft(B, kind, Hq, Hkv, d, n_old, n_new, seed=33, append=False)
    places = [(b % Hkv, a + m // 2) if b % 2 == 0 and m else None for b, (a, m) in enumerate(zip(n_old, n_new))]
    for b, place in enumerate(places):
        if place:
            h, slot = place
            x.k_new[b, slot - n_old[b], h, 5] = math.nan
            x.K[b, h, slot] = 0
    x.v_new[x.v_new.isnan()] = 0.0
    B.dynts_chunk_step(x.c.ctx, 0, x.q.to(DEV), x.k_new, x.v_new, x.out, x.scratch, lse=x.lse, n_new=x.n)
    for b, (a, m) in enumerate(zip(n_old, n_new)):
        r, rows, slots = _attend(x, b, places[b])
        _check(x.out[b, :m], r["out"], r["out_tol"], rows[:, :, None], "out[%d]" % b)
        _check(x.lse[b, :m], r["lse"], r["lse_tol"], rows, "lse[%d]" % b)
        _check(x.c.S[0, b, :, :a + m], r["recv"], r["recv_tol"], slots, "received[%d]" % b)
    assert int(x.c.status.item()) == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("Hq,Hkv,d,n_old,n_new", SHAPES)
def test_values(B, kind, Hq, Hkv, d, n_old, n_new):
    """A NaN in a row of V: in that element (on codes its block) of the tokens that see the row, and in none of the others' elements, lse and weights.  (That element of
    tokens that do not see the row, those before it in the same chunk, is not told: hidden rows of V have to be finite.)"""
    x = Draft(B, kind, Hq, Hkv, d, n_old, n_new, seed=34, append=False)
    x.k_new[x.k_new.isnan()] = 0.0
    x.v_new[x.v_new.isnan()] = 0.0
    places = [(b % Hkv, m // 2) if m else None for b, m in enumerate(n_new)]
    elements = torch.zeros(d, dtype=torch.bool)
    if _code(kind):
        elements[32:64] = True
    else:
        elements[37] = True
    for b, place in enumerate(places):
        if place:
            h, at = place
            x.v_new[b, at, h, 37] = math.nan
            x.V[b, h, n_old[b] + at, elements] = 0  # (of what it is compared with, these elements are left out)
    B.dynts_chunk_step(x.c.ctx, 0, x.q.to(DEV), x.k_new, x.v_new, x.out, x.scratch, lse=x.lse, n_new=x.n)
    G = Hq // Hkv
    for b, (a, m) in enumerate(zip(n_old, n_new)):
        r, rows, slots = _attend(x, b, None)
        _check(x.lse[b, :m], r["lse"], r["lse_tol"], rows, "lse[%d]" % b)
        _check(x.c.S[0, b, :, :a + m], r["recv"], r["recv_tol"], slots, "received[%d]" % b)
        rest = torch.ones((m, Hq, d), dtype=torch.bool)
        if places[b]:
            h, at = places[b]
            heads = slice(h * G, (h + 1) * G)
            assert torch.all(x.out[b, at:m, heads][:, :, elements.to(DEV)].isnan())
            rest[:, heads] = ~elements
        plain.check(x.out[b, :m].double().cpu()[rest], r["out"][rest], r["out_tol"][rest], "out[%d]" % b)
    assert int(x.c.status.item()) == 0
