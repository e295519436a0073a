"""What the binding of the chunk entry points knows of a context's arrays, no GPU needed."""
import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2601_18383_amd import binding, build
    if build.is_stale():
        build.build()
    return binding


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


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("cache_gpu,current", [(0, 0), (1, 1), (1, 0), (0, 1), (-1, 0)])
def test_a_cache_of_another_gpu_is_refused(B, monkeypatch, paged, cache_gpu, current):
    """Bound by dynts_bind or dynts_bind_paged on one GPU, called with tensors of the current one: no call of the library may follow."""
    import torch
    called = []
    for name in ("dynts_bind", "dynts_bind_paged"):
        monkeypatch.setattr(B.lib, name, lambda *a: B.DYNTS_OK)
    for name in ("append", "attend", "scores", "step"):
        monkeypatch.setattr(B.lib, "dynts_chunk_" + name, lambda *a, name=name: called.append(name) or B.DYNTS_OK)
    monkeypatch.setattr(B, "_device", lambda: current)
    monkeypatch.setattr(B, "_stream", lambda s: None)
    Nb, Hq, Hkv, d, cap, T = 3, 8, 2, 128, 400, 5
    ctx = B.dynts_create(B.make_config(1, Nb, Hq, Hkv, d, cap, 0, 0, 1))
    bf16, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    t = lambda dtype, *shape: On(cache_gpu, dtype, *shape)
    rest = [t(f32, 1, Nb, Hkv, cap), t(i32, 1, Nb, Hkv, cap), t(i32, 1, Nb), t(i32, 1, Nb), t(i32, Nb), t(torch.uint8, 4096), t(i32, 1)]
    if paged:
        pool = t(bf16, 50, 64, d)
        B.dynts_bind_paged(ctx, pool, pool, t(i32, 1, Nb, Hkv, 7), t(i32, 50), t(i32, 1), *rest)
    else:
        K = t(bf16, 1, Nb, Hkv, cap, d)
        B.dynts_bind(ctx, K, K, *rest)
    here = lambda dtype, *shape: On(current, dtype, *shape)
    q, k, lse, s = here(bf16, Nb, T, Hq, d), here(bf16, Nb, T, Hkv, d), here(f32, Nb, T, Hq), here(torch.uint8, 4096)
    calls = [lambda: B.dynts_chunk_append(ctx, 0, k, k, s), lambda: B.dynts_chunk_attend(ctx, 0, q, q, s), lambda: B.dynts_chunk_scores(ctx, 0, q, lse),
             lambda: B.dynts_chunk_step(ctx, 0, q, k, k, q, s)]
    for call in calls:
        if cache_gpu == current:
            call()
        else:
            with pytest.raises(ValueError):
                call()
    assert called == (["append", "attend", "scores", "step"] if cache_gpu == current else [])
    B.dynts_destroy(ctx)


def test_a_cache_bound_by_addresses_is_the_callers_affair(B, monkeypatch):
    """Bare addresses say nothing of where they lie; a context bound again forgets where the last arrays lay."""
    import torch
    monkeypatch.setattr(B.lib, "dynts_bind", lambda *a: B.DYNTS_OK)
    monkeypatch.setattr(B, "_device", lambda: 0)
    ctx = B.dynts_create(B.make_config(1, 1, 8, 2, 128, 400, 0, 0, 1))
    K, ws = On(1, torch.bfloat16, 1, 1, 2, 400, 128), On(1, torch.uint8, 4096)
    B.dynts_bind(ctx, K, K, *([256] * 5), ws, 256)
    q = On(0, torch.bfloat16, 1, 5, 8, 128)
    with pytest.raises(ValueError):
        B._on_device(ctx, q)
    B.dynts_bind(ctx, 256, 256, *([256] * 5), ws, 256)
    B._on_device(ctx, q)
    B.dynts_destroy(ctx)
