"""Host side of caches of codes and of drafts, no GPU needed: every refusal comes before any launch."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2601_18383_amd import binding, build
    if build.is_stale():
        build.build()
    return binding


def _cfg(B, **kw):
    base = dict(n_layers=2, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=128, capacity=400, budget=256, window=64,
                evict_every=16, softmax_scale=0.0, score_mode=0)
    base.update(kw)
    return B.make_config(**base)


ONE = C.c_void_p(256)  # non-null and aligned, never dereferenced: the checks fail first
ODD = C.c_void_p(264)
FAR = C.c_void_p(1 << 40)
BIG = C.c_void_p(1 << 41)


def _codes(B, **kw):
    x = dict(code=B.DYNTS_CODE_INT8, K=256, V=256, K_scale=256, V_scale=256, n_pages=0, max_pages=0, block_table=None, free_stack=None, free_top=None)
    x.update(kw)
    return B.dynts_codes(*[x[n] for n, _ in B.dynts_codes._fields_])


def _bind(B, ctx, cfg, codes, ws=ONE):
    return B.lib.dynts_bind_codes(ctx, C.byref(codes) if codes else None, *([ONE] * 5), ws, B.dynts_workspace_bytes(cfg), ONE)


def _bound(B, coded=True, **kw):
    cfg = _cfg(B, **kw)
    ctx = B.dynts_create(cfg)
    if coded:
        assert _bind(B, ctx, cfg, _codes(B)) == B.DYNTS_OK
    else:
        assert B.lib.dynts_bind(ctx, *([ONE] * 7), ONE, B.dynts_workspace_bytes(cfg), ONE) == B.DYNTS_OK
    return cfg, ctx


def test_bind_refusals(B):
    cfg = _cfg(B)
    ctx = B.dynts_create(cfg)
    assert _bind(B, None, cfg, _codes(B)) == B.DYNTS_ENULL
    assert _bind(B, ctx, cfg, None) == B.DYNTS_ENULL
    for name in ("K", "V", "K_scale", "V_scale"):
        assert _bind(B, ctx, cfg, _codes(B, **{name: None})) == B.DYNTS_ENULL
        assert _bind(B, ctx, cfg, _codes(B, **{name: 264})) == B.DYNTS_EINVAL
    for code in (0, 3, -1):
        assert _bind(B, ctx, cfg, _codes(B, code=code)) == B.DYNTS_EINVAL
    assert _bind(B, ctx, cfg, _codes(B), ws=ODD) == B.DYNTS_EWORKSPACE
    pages = dict(block_table=256, free_stack=256, free_top=256, n_pages=100, max_pages=7)
    assert _bind(B, ctx, cfg, _codes(B, **dict(pages, max_pages=6))) == B.DYNTS_ECAPACITY
    assert _bind(B, ctx, cfg, _codes(B, **dict(pages, free_top=None))) == B.DYNTS_ENULL
    assert _bind(B, ctx, cfg, _codes(B, **dict(pages, n_pages=0))) == B.DYNTS_EINVAL
    # none of them has bound anything
    assert B.lib.dynts_read_rows(ctx, 0, None, 1, ONE, FAR, None) == B.DYNTS_ENOTBOUND
    assert _bind(B, ctx, cfg, _codes(B, **pages)) == B.DYNTS_OK
    B.dynts_destroy(ctx)


def test_calls_for_bf16_caches_say_so(B):
    L = B.lib
    cfg, ctx = _bound(B)

    def calls():
        return [L.dynts_prefill(ctx, 0, None, ONE, 4, ONE, None), L.dynts_append(ctx, 0, None, ONE, None, None, None),
                L.dynts_decode_attend(ctx, 0, None, None, ONE, None, None), L.dynts_decode_attend_update(ctx, 0, None, None, ONE, None, None),
                L.dynts_decode_step(ctx, 0, None, ONE, ONE, None, None, ONE, None, None),
                L.dynts_decode_step_static(ctx, 0, None, ONE, ONE, None, None, ONE, None, None),
                L.dynts_score_block(ctx, 0, None, None, 4, None, None, 1, ONE, 1 << 30, None),
                L.dynts_decode_loop(ctx, 1, None, ONE, ONE, None, None, None, None, ONE, 0, None, None, None)]
    assert set(calls()) == {B.DYNTS_ECODES}
    assert L.dynts_hint_trigger(ctx, 0) == B.DYNTS_ECODES
    assert "codes" in B.dynts_strerror(B.DYNTS_ECODES)
    assert L.dynts_update_scores(ctx, 0, None) == B.DYNTS_OK  # (nothing is owed, nothing is launched)
    # bound to a bf16 cache again, the context takes them again: null arguments are what they find
    assert L.dynts_bind(ctx, *([ONE] * 7), ONE, B.dynts_workspace_bytes(cfg), ONE) == B.DYNTS_OK
    assert set(calls()) == {B.DYNTS_ENULL} and L.dynts_hint_trigger(ctx, 0) == B.DYNTS_OK
    B.dynts_destroy(ctx)


def test_scratch_sizes(B):
    for kw in (dict(), dict(batch=1, capacity=100000), dict(batch=128, n_q_heads=28, n_kv_heads=4), dict(head_dim=64, batch=5)):
        cfg, last = _cfg(B, **kw), 0
        for t in list(range(1, 300)) + [1000, 5000, 1 << 20]:
            size = B.dynts_codes_scratch_bytes(cfg, t)
            assert size >= max(last, B.dynts_chunk_scratch_bytes(cfg, t)), (kw, t)
            last = size
        # many rows: one layer's rows as bf16 fit
        assert last >= B.dynts_chunk_scratch_bytes(cfg, 1 << 20) + 2 * 2 * cfg.batch * cfg.n_kv_heads * cfg.capacity * cfg.head_dim
    for t in (0, -1, (1 << 20) + 1):
        assert B.dynts_codes_scratch_bytes(_cfg(B), t) == 0
    assert B.dynts_codes_scratch_bytes(_cfg(B, head_dim=96), 4) == 0 and B.lib.dynts_codes_scratch_bytes(None, 4) == 0


def test_chunks_on_codes_want_their_own_scratch(B):
    L = B.lib
    cfg, ctx = _bound(B, batch=64, n_q_heads=32, n_kv_heads=8)
    T = 64
    small, need = B.dynts_chunk_scratch_bytes(cfg, T), B.dynts_codes_scratch_bytes(cfg, T)
    assert small < need
    for size in (small, need - 1):
        assert L.dynts_chunk_attend(ctx, 0, ONE, T, None, None, FAR, None, ONE, size, None) == B.DYNTS_EWORKSPACE
        assert L.dynts_chunk_append(ctx, 0, ONE, ONE, None, T, None, 0, ONE, size, None) == B.DYNTS_EWORKSPACE
        assert L.dynts_chunk_step(ctx, 0, ONE, ONE, ONE, None, T, None, 0, None, FAR, None, ONE, size, None) == B.DYNTS_EWORKSPACE
        assert L.dynts_tree_attend(ctx, 0, ONE, T, None, ONE, FAR, None, ONE, size, None) == B.DYNTS_EWORKSPACE
        assert L.dynts_tree_step(ctx, 0, ONE, ONE, ONE, None, T, None, ONE, ONE, FAR, None, ONE, size, None) == B.DYNTS_EWORKSPACE
    B.dynts_destroy(ctx)


@pytest.mark.parametrize("coded", [False, True])
def test_read_rows_refusals(B, coded):
    cfg, ctx = _bound(B, coded)
    f = B.lib.dynts_read_rows
    assert f(None, 0, None, 4, ONE, FAR, None) == B.DYNTS_ENULL
    assert f(ctx, 2, None, 4, ONE, FAR, None) == B.DYNTS_EINVAL and f(ctx, -1, None, 4, ONE, FAR, None) == B.DYNTS_EINVAL
    assert f(ctx, 0, None, 4, None, FAR, None) == B.DYNTS_ENULL and f(ctx, 0, None, 4, ONE, None, None) == B.DYNTS_ENULL
    for n in (0, -1, 401):
        assert f(ctx, 0, None, n, ONE, FAR, None) == B.DYNTS_EINVAL
    assert f(ctx, 0, None, 4, ODD, FAR, None) == B.DYNTS_EINVAL and f(ctx, 0, C.c_void_p(258), 4, ONE, FAR, None) == B.DYNTS_EINVAL
    assert f(ctx, 0, None, 4, ONE, C.c_void_p(256 + 3 * 2 * 4 * 128 * 2 - 16), None) == B.DYNTS_EINVAL  # overlap
    B.dynts_destroy(ctx)


def test_tree_build_refusals(B):
    f = B.lib.dynts_tree_build
    assert f(None, None, 2, 4, FAR, None, None) == B.DYNTS_ENULL and f(ONE, None, 2, 4, None, None, None) == B.DYNTS_ENULL
    for batch, T in ((0, 4), (-1, 4), (65536, 4), (2, 0), (2, -5), (2, 4097)):
        assert f(ONE, None, batch, T, FAR, None, None) == B.DYNTS_EINVAL
    bad = C.c_void_p(258)
    assert f(bad, None, 2, 4, FAR, None, None) == B.DYNTS_EINVAL and f(ONE, bad, 2, 4, FAR, None, None) == B.DYNTS_EINVAL
    assert f(ONE, None, 2, 4, C.c_void_p((1 << 40) + 2), None, None) == B.DYNTS_EINVAL
    assert f(ONE, None, 2, 4, ONE, None, None) == B.DYNTS_EINVAL  # over the parents
    assert f(ONE, None, 2, 4, FAR, ONE, None) == B.DYNTS_EINVAL and f(ONE, None, 2, 4, FAR, FAR, None) == B.DYNTS_EINVAL


@pytest.mark.parametrize("coded", [False, True])
def test_draft_refusals(B, coded):
    L = B.lib
    cfg, ctx = _bound(B, coded)
    T = 16
    need = B.dynts_codes_scratch_bytes(cfg, T)
    base = dict(ctx=ctx, layer=0, q=ONE, T=T, n=None, seen=ONE, out=FAR, lse=None, scratch=ONE, size=need, k=ONE, v=ONE, s=None, taken=ONE, leaf=ONE,
                kept=C.c_void_p(512), q_kept=None, lse_kept=None)

    def attend(**kw):
        x = dict(base, **kw)
        return L.dynts_tree_attend(x["ctx"], x["layer"], x["q"], x["T"], x["n"], x["seen"], x["out"], x["lse"], x["scratch"], x["size"], None)

    def step(**kw):
        x = dict(base, **kw)
        return L.dynts_tree_step(x["ctx"], x["layer"], x["q"], x["k"], x["v"], x["s"], x["T"], x["n"], x["seen"], x["taken"], x["out"], x["lse"],
                                 x["scratch"], x["size"], None)

    def keep(**kw):
        x = dict(base, **kw)
        return L.dynts_tree_keep(x["ctx"], x["layer"], x["T"], x["n"], x["seen"], x["leaf"], x["q"], x["lse"], x["q_kept"], x["lse_kept"], x["kept"], None)

    for f in (attend, step, keep):
        assert f(ctx=None) == B.DYNTS_ENULL and f(seen=None) == B.DYNTS_ENULL
        assert f(layer=2) == B.DYNTS_EINVAL and f(layer=-1) == B.DYNTS_EINVAL
        assert f(seen=C.c_void_p(258)) == B.DYNTS_EINVAL
        for t in (0, -1, 4097):
            assert f(T=t) == B.DYNTS_EINVAL
    for f in (attend, step):
        assert f(q=None) == B.DYNTS_ENULL and f(out=None) == B.DYNTS_ENULL and f(scratch=None) == B.DYNTS_ENULL
        assert f(q=ODD) == B.DYNTS_EINVAL and f(out=ODD) == B.DYNTS_EINVAL and f(out=ONE) == B.DYNTS_EINVAL
        assert f(scratch=ODD) == B.DYNTS_EWORKSPACE and f(size=B.dynts_chunk_scratch_bytes(cfg, T) - 1) == B.DYNTS_EWORKSPACE
    assert step(k=None) == B.DYNTS_ENULL and step(v=None) == B.DYNTS_ENULL and step(taken=None) == B.DYNTS_ENULL
    assert step(k=ODD) == B.DYNTS_EINVAL and step(v=ODD) == B.DYNTS_EINVAL
    assert step(k=FAR) == B.DYNTS_EINVAL and step(v=FAR) == B.DYNTS_EINVAL  # out over them
    assert keep(leaf=None) == B.DYNTS_ENULL and keep(kept=None) == B.DYNTS_ENULL
    assert keep(q_kept=FAR, q=None) == B.DYNTS_ENULL and keep(lse_kept=FAR, lse=None) == B.DYNTS_ENULL
    assert keep(q_kept=ONE) == B.DYNTS_EINVAL and keep(lse_kept=ONE, lse=ONE) == B.DYNTS_EINVAL
    assert keep(q_kept=C.c_void_p((1 << 40) + 8)) == B.DYNTS_EINVAL
    assert keep(kept=ONE) == B.DYNTS_EINVAL and keep(leaf=FAR, n=ONE, kept=C.c_void_p(264)) == B.DYNTS_EINVAL  # over leaf, over n_taken
    B.dynts_destroy(ctx)
    ctx = B.dynts_create(cfg)
    assert attend(ctx=ctx) == B.DYNTS_ENOTBOUND and step(ctx=ctx) == B.DYNTS_ENOTBOUND and keep(ctx=ctx) == B.DYNTS_ENOTBOUND
    B.dynts_destroy(ctx)
    cfg, ctx = _bound(B, coded, score_mode=1)
    assert step(ctx=ctx) == B.DYNTS_ENULL  # scores from outside have to be given
    B.dynts_destroy(ctx)


class On:
    """A tensor of one GPU, as far as the binding looks at it."""

    def __init__(self, gpu, dtype, *shape):
        self.gpu, self.dtype, self.shape = gpu, dtype, shape

    def get_device(self):
        return self.gpu

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 256

    def element_size(self):
        return 1

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n


def test_tensors_elsewhere_or_of_other_sizes_are_refused(B, monkeypatch):
    import torch
    called = []
    for name in ("read_rows", "tree_build", "tree_attend", "tree_step", "tree_keep"):
        monkeypatch.setattr(B.lib, "dynts_" + name, lambda *a, name=name: called.append(name) or B.DYNTS_OK)
    monkeypatch.setattr(B.lib, "dynts_bind_codes", lambda *a: B.DYNTS_OK)
    monkeypatch.setattr(B, "_device", lambda: 0)
    monkeypatch.setattr(B, "_stream", lambda s: None)
    Nb, Hq, Hkv, d, cap, T = 3, 8, 2, 128, 400, 40
    bf16, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8

    def context(gpu):
        ctx = B.dynts_create(B.make_config(1, Nb, Hq, Hkv, d, cap, 0, 0, 1))
        t = lambda dtype, *shape: On(gpu, dtype, *shape)
        codes, scale = t(u8, 1, Nb, Hkv, cap, d), t(u8, 1, Nb, Hkv, cap, d // 32)
        B.dynts_bind_codes(ctx, B.DYNTS_CODE_INT8, codes, codes, scale, scale, t(f32, 1), t(i32, 1), t(i32, 1), t(i32, 1), t(i32, 1), t(u8, 4096), t(i32, 1))
        return ctx

    def calls(ctx, gpu=0, T2=T, W=2, heads=Hkv, n=Nb):
        t = lambda dtype, *shape: On(gpu, dtype, *shape)
        q, k, rows = t(bf16, Nb, T, Hq, d), t(bf16, Nb, T2, heads, d), t(bf16, Nb, heads, 9, d)
        seen, lse, s, one = t(i32, Nb, T, W), t(f32, Nb, T2, Hq), t(u8, 4096), t(i32, n)
        return [lambda: B.dynts_read_rows(ctx, 0, rows, rows, first=one), lambda: B.dynts_tree_build(t(i32, Nb, T2), seen, depth=t(i32, Nb, T), n_new=one),
                lambda: B.dynts_tree_attend(ctx, 0, q, seen, q, s, lse=lse, n_new=one),
                lambda: B.dynts_tree_step(ctx, 0, q, k, k, seen, one, q, s, lse=lse, n_new=one),
                lambda: B.dynts_tree_keep(ctx, 0, seen, one, one, one, q=q, lse=lse, q_kept=q, lse_kept=lse)]

    ctx = context(0)
    for call in calls(ctx):
        call()
    assert len(called) == 5
    for kw in (dict(gpu=1), dict(gpu=-1)):
        for call in calls(ctx, **kw):
            with pytest.raises(ValueError):
                call()
    for call in calls(ctx, T2=T + 1)[1:]:
        with pytest.raises(AssertionError):
            call()
    for call in calls(ctx, W=1)[1:] + calls(ctx, n=Nb + 1):
        with pytest.raises(AssertionError):
            call()
    for i in (0, 3):
        with pytest.raises(AssertionError):
            calls(ctx, heads=4)[i]()
    there = context(1)
    for i in (0, 2, 3, 4):  # a cache of another GPU
        with pytest.raises(ValueError):
            calls(there)[i]()
    assert len(called) == 5
    B.dynts_destroy(ctx)
    B.dynts_destroy(there)


def test_a_row_finds_its_token():
    """The multiplication that stands for the division of rows by heads: exact at every border of up to 2^20 tokens of up to 128 heads."""
    for heads in range(1, 129):
        magic = ((1 << 36) + heads - 1) // heads
        for token in [0, 1, 2, 1000, 304000, 304001, (1 << 19) + 1, (1 << 20) - 1]:
            for row in (token * heads, token * heads + heads - 1):
                assert row < 1 << 27 and row * magic >> 36 == token and row * magic < 1 << 64
