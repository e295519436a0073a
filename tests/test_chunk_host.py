"""Host side of the chunk and rotary entry points, no GPU needed: every refusal comes before any launch."""
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


def _bound(B, **kw):
    cfg = _cfg(B, **kw)
    ctx = B.dynts_create(cfg)
    assert B.lib.dynts_bind(ctx, *([ONE] * 7), ONE, B.dynts_workspace_bytes(cfg), ONE) == B.DYNTS_OK
    return cfg, ctx


def test_scratch_sizes(B):
    cfg = _cfg(B)
    sizes = [B.dynts_chunk_scratch_bytes(cfg, t) for t in (1, 2, 5, 16, 64, 100, 1000, 1 << 20)]
    assert all(s > 0 for s in sizes) and sizes == sorted(sizes)
    for t in (0, -1, (1 << 20) + 1):
        assert B.dynts_chunk_scratch_bytes(cfg, t) == 0
    assert B.dynts_chunk_scratch_bytes(_cfg(B, head_dim=96), 4) == 0
    assert B.lib.dynts_chunk_scratch_bytes(None, 4) == 0


def test_what_serves_a_chunk_serves_every_smaller_one(B):
    for kw in (dict(), dict(batch=1, capacity=100000), dict(batch=128, n_q_heads=28, n_kv_heads=4), dict(head_dim=64, batch=5)):
        cfg, last = _cfg(B, **kw), 0
        for t in range(1, 700):
            size = B.dynts_chunk_scratch_bytes(cfg, t)
            assert size >= last, (kw, t)
            last = size


def test_chunk_refusals(B):
    L = B.lib
    cfg, ctx = _bound(B)
    T = 16
    need = B.dynts_chunk_scratch_bytes(cfg, T)
    attend = dict(ctx=ctx, layer=0, q=ONE, T=T, n=None, sh=None, out=ONE, lse=None, scratch=ONE, size=need)

    def a(**kw):
        x = dict(attend, **kw)
        return L.dynts_chunk_attend(x["ctx"], x["layer"], x["q"], x["T"], x["n"], x["sh"], x["out"], x["lse"], x["scratch"], x["size"], None)

    def s(**kw):
        x = dict(attend, lse=ONE, **kw)
        return L.dynts_chunk_scores(x["ctx"], x["layer"], x["q"], x["T"], x["n"], x["sh"], x["lse"], None, 1, None)

    def step(**kw):
        x = dict(attend, k=ONE, v=ONE, s=None, question=0, **kw)
        return L.dynts_chunk_step(x["ctx"], x["layer"], x["q"], x["k"], x["v"], x["s"], x["T"], x["n"], x["question"], x["sh"], x["out"], x["lse"],
                                  x["scratch"], x["size"], None)

    def app(**kw):
        x = dict(attend, k=ONE, v=ONE, s=None, question=0)
        x.update(kw)
        return L.dynts_chunk_append(x["ctx"], x["layer"], x["k"], x["v"], x["s"], x["T"], x["n"], x["question"], x["scratch"], x["size"], None)

    odd = C.c_void_p(264)
    bad_shapings = [B.dynts_shaping(-1.0, 0, None, None, None), B.dynts_shaping(float("nan"), 0, None, None, None),
                    B.dynts_shaping(float("inf"), 0, None, None, None), B.dynts_shaping(0.0, -1, None, None, None),
                    B.dynts_shaping(0.0, 0, 258, None, None), B.dynts_shaping(0.0, 0, None, 257, None), B.dynts_shaping(0.0, 0, None, None, 259)]
    for f in (a, s, step):
        assert f(ctx=None) == B.DYNTS_ENULL
        assert f(layer=2) == B.DYNTS_EINVAL and f(layer=-1) == B.DYNTS_EINVAL
        assert f(T=0) == B.DYNTS_EINVAL and f(T=(1 << 20) + 1) == B.DYNTS_EINVAL
        assert f(q=None) == B.DYNTS_ENULL and f(q=odd) == B.DYNTS_EINVAL
        for sh in bad_shapings:
            assert f(sh=C.byref(sh)) == B.DYNTS_EINVAL
    for f in (a, step):
        assert f(out=None) == B.DYNTS_ENULL and f(out=odd) == B.DYNTS_EINVAL
    for f in (a, step, app):
        assert f(scratch=None) == B.DYNTS_ENULL
        assert f(scratch=odd) == B.DYNTS_EWORKSPACE and f(size=need - 1) == B.DYNTS_EWORKSPACE
    assert app(ctx=None) == B.DYNTS_ENULL and app(layer=7) == B.DYNTS_EINVAL and app(T=0) == B.DYNTS_EINVAL
    assert app(k=None) == B.DYNTS_ENULL and app(v=None) == B.DYNTS_ENULL
    assert app(k=odd) == B.DYNTS_EINVAL and app(v=odd) == B.DYNTS_EINVAL
    x = dict(attend)
    assert L.dynts_chunk_scores(ctx, 0, ONE, T, None, None, None, None, 1, None) == B.DYNTS_ENULL
    assert L.dynts_chunk_step(ctx, 0, ONE, None, ONE, None, T, None, 0, None, ONE, None, ONE, need, None) == B.DYNTS_ENULL
    assert L.dynts_chunk_step(ctx, 0, ONE, ONE, odd, None, T, None, 0, None, ONE, None, ONE, need, None) == B.DYNTS_EINVAL
    B.dynts_destroy(ctx)
    # not bound; scores from outside have to be given, but not for question tokens (that call would launch: not made here)
    ctx = B.dynts_create(cfg)
    assert L.dynts_chunk_attend(ctx, 0, ONE, T, None, None, ONE, None, ONE, need, None) == B.DYNTS_ENOTBOUND
    assert L.dynts_chunk_append(ctx, 0, ONE, ONE, None, T, None, 0, ONE, need, None) == B.DYNTS_ENOTBOUND
    assert L.dynts_chunk_scores(ctx, 0, ONE, T, None, None, ONE, None, 1, None) == B.DYNTS_ENOTBOUND
    assert L.dynts_chunk_step(ctx, 0, ONE, ONE, ONE, None, T, None, 0, None, ONE, None, ONE, need, None) == B.DYNTS_ENOTBOUND
    B.dynts_destroy(ctx)
    cfg, ctx = _bound(B, score_mode=1)
    assert L.dynts_chunk_append(ctx, 0, ONE, ONE, None, T, None, 0, ONE, need, None) == B.DYNTS_ENULL
    assert L.dynts_chunk_step(ctx, 0, ONE, ONE, ONE, None, T, None, 0, None, ONE, None, ONE, need, None) == B.DYNTS_ENULL
    B.dynts_destroy(ctx)


def test_grids_past_their_limit_are_refused(B):
    # 8192 sequences of 128 heads and a million tokens each: more workgroups than a grid holds
    cfg, ctx = _bound(B, batch=65535, n_q_heads=1024, n_kv_heads=64, head_dim=128, capacity=1 << 22)
    T = 1 << 20
    need = B.dynts_chunk_scratch_bytes(cfg, T)
    assert B.lib.dynts_chunk_attend(ctx, 0, ONE, T, None, None, ONE, None, ONE, need, None) == B.DYNTS_EINVAL
    assert B.lib.dynts_chunk_scores(ctx, 0, ONE, T, None, None, ONE, None, 1, None) == B.DYNTS_EINVAL
    assert B.lib.dynts_chunk_step(ctx, 0, ONE, ONE, ONE, None, T, None, 0, None, ONE, None, ONE, need, None) == B.DYNTS_EINVAL
    B.dynts_destroy(ctx)


def test_an_output_over_an_input_is_refused(B):
    cfg, ctx = _bound(B)
    T, at = 16, lambda x: C.c_void_p(1 << 30 | x)
    need, rows, k_rows = B.dynts_chunk_scratch_bytes(cfg, T), 3 * T * 8 * 128 * 2, 3 * T * 2 * 128 * 2
    far, scratch = at(1 << 28), at(1 << 29)
    for out in (at(0), at(16), at(rows - 16)):
        assert B.lib.dynts_chunk_attend(ctx, 0, at(0), T, None, None, out, None, scratch, need, None) == B.DYNTS_EINVAL
        assert B.lib.dynts_chunk_attend(ctx, 0, out, T, None, None, at(0), None, scratch, need, None) == B.DYNTS_EINVAL
    for out in (at(0), at(k_rows - 16)):
        assert B.lib.dynts_chunk_step(ctx, 0, far, at(0), far, None, T, None, 0, None, out, None, scratch, need, None) == B.DYNTS_EINVAL
        assert B.lib.dynts_chunk_step(ctx, 0, far, far, at(0), None, T, None, 0, None, out, None, scratch, need, None) == B.DYNTS_EINVAL
    B.dynts_destroy(ctx)


def test_rotate_refusals(B):
    L = B.lib

    def r(d=128, pairs=64, pairing=0, axes=1, freq=256, axis=None, q=ONE, hq=4, k=ONE, hk=2, pos=ONE, n=3, qo=ONE, ko=ONE):
        t = B.dynts_rotary(d, pairs, pairing, axes, freq, axis)
        return L.dynts_rotate(C.byref(t), q, hq, k, hk, pos, n, 0, qo, ko, None)

    assert L.dynts_rotate(None, ONE, 4, ONE, 2, ONE, 3, 0, ONE, ONE, None) == B.DYNTS_ENULL
    assert r(pairing=2) == B.DYNTS_EINVAL and r(pairing=-1) == B.DYNTS_EINVAL
    assert r(axes=0) == B.DYNTS_EINVAL and r(pairs=0) == B.DYNTS_EINVAL and r(n=-1) == B.DYNTS_EINVAL
    for kw in (dict(d=0), dict(d=-8), dict(d=100), dict(pairs=12), dict(pairs=72), dict(d=512, pairs=136), dict(d=64, pairs=40),
               dict(hq=1 << 22), dict(n=1 << 24)):
        assert r(**kw) == B.DYNTS_ESHAPE, kw
    for kw in (dict(freq=None), dict(pos=None), dict(q=None), dict(qo=None), dict(ko=None)):
        assert r(**kw) == B.DYNTS_ENULL, kw
    odd = C.c_void_p(264)
    for kw in (dict(q=odd), dict(qo=odd), dict(k=odd), dict(ko=odd), dict(hq=0), dict(hk=0), dict(hk=-1)):
        assert r(**kw) == B.DYNTS_EINVAL, kw
    assert r(n=0) == B.DYNTS_OK  # nothing to turn: no launch


def test_the_binding_refuses_what_does_not_fit(B):
    """Tensors of the host, sizes that do not belong together: found before the library is called."""
    import torch
    ctx = C.c_void_p(0)  # (a call that came through would be answered with an error for it)
    q = torch.zeros((2, 3, 8, 64), dtype=torch.bfloat16)
    k = torch.zeros((2, 3, 2, 64), dtype=torch.bfloat16)
    lse = torch.zeros((2, 3, 8))
    s = torch.zeros(64, dtype=torch.uint8)
    n2, n3 = torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    pos = torch.zeros((2, 4), dtype=torch.int32)
    for call in (lambda: B.dynts_chunk_attend(ctx, 0, q, q, s), lambda: B.dynts_chunk_scores(ctx, 0, q, lse),
                 lambda: B.dynts_chunk_step(ctx, 0, q, k, k, q, s), lambda: B.dynts_chunk_append(ctx, 0, k, k, s),
                 lambda: B.dynts_rotate(B.Rotary(64, torch.ones(32)), q, k, torch.zeros((1, 2, 3), dtype=torch.int32), q, k)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.dynts_chunk_attend(ctx, 0, q, q, s, n_new=n3), lambda: B.dynts_chunk_attend(ctx, 0, q, q, s, lse=lse[:1]),
                 lambda: B.dynts_chunk_attend(ctx, 0, q, q, s, shaping=B.Shaping(first=pos)),
                 lambda: B.dynts_chunk_attend(ctx, 0, q, q, s, shaping=B.Shaping(last=pos)),
                 lambda: B.dynts_chunk_scores(ctx, 0, q, lse, shaping=B.Shaping(slope=torch.zeros(7))),
                 lambda: B.dynts_chunk_append(ctx, 0, k, k[:, :2], s), lambda: B.dynts_chunk_append(ctx, 0, k, q, s),
                 lambda: B.dynts_rotate(B.Rotary(64, torch.ones(32)), q, k, torch.zeros((1, 2, 4), dtype=torch.int32), q, k),
                 lambda: B.dynts_rotate(B.Rotary(64, torch.ones(32)), q, k, torch.zeros((1, 2, 3), dtype=torch.int32), q, q),
                 lambda: B.Rotary(64, torch.ones(32), axis=torch.zeros(31, dtype=torch.uint8)),
                 lambda: B.Shaping(first=torch.zeros((2, 3))), lambda: B.Shaping(slope=torch.zeros((8, 2))[:, 0])):
        with pytest.raises(AssertionError):
            call()
    assert n2.numel() == 2


def test_the_binding_refuses_a_cache_of_another_gpu(B, monkeypatch):
    class OnGpu:
        def get_device(self):
            return 0

    monkeypatch.setattr(B, "_device", lambda: 0)
    ctx = C.c_void_p(0)
    B._on_device(ctx, OnGpu(), None)
    ctx.gpu = 0
    B._on_device(ctx, OnGpu(), None)
    ctx.gpu = 1
    with pytest.raises(ValueError):
        B._on_device(ctx, OnGpu(), None)
    monkeypatch.setattr(B, "_device", lambda: 1)
    with pytest.raises(ValueError):
        B._on_device(ctx, OnGpu(), None)


def test_the_binding_refuses_chunks_of_another_context(B):
    """Batch, heads and head_dim of the context, and the size of dst: a smaller tensor would be read or written past its end."""
    import torch
    cfg, ctx = _bound(B)  # 3 sequences, 8 heads on 2 of 128, 400 slots
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    q, k, s = z(3, 5, 8, 128), z(3, 5, 2, 128), torch.zeros(64, dtype=torch.uint8)
    lse = torch.zeros((3, 5, 8))
    for bad in (z(2, 5, 8, 128), z(3, 5, 4, 128), z(3, 5, 8, 64)):
        with pytest.raises(AssertionError):
            B.dynts_chunk_attend(ctx, 0, bad, bad, s)
        with pytest.raises(AssertionError):
            B.dynts_chunk_step(ctx, 0, bad, k, k, bad, s)
    for bad in (z(2, 5, 2, 128), z(3, 5, 1, 128), z(3, 5, 2, 64)):
        with pytest.raises(AssertionError):
            B.dynts_chunk_append(ctx, 0, bad, bad, s)
    with pytest.raises(AssertionError):
        B.dynts_chunk_scores(ctx, 0, q, lse, dst=torch.zeros((3, 2, 399)))
    with pytest.raises(ValueError):  # (these sizes fit: it is the host's tensors that are refused)
        B.dynts_chunk_scores(ctx, 0, q, lse, dst=torch.zeros((3, 2, 400)))
    rot = B.Rotary(128, torch.ones(64))
    assert rot.gpu < 0  # tables of the host are refused wherever the queries are
    B.dynts_destroy(ctx)
