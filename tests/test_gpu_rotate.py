"""Rotary positions (dynts_rotate) against the definition in float64; the gradient against the formula's and against differences."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def B():
    from paper_2601_18383_amd import binding
    return binding


def turn(x, positions, freq, axis, adjacent, inverse=False):
    """x [tokens][heads][d] -> float64."""
    P = freq.numel()
    y = x.double().clone()
    a = axis.long() if axis is not None else torch.zeros(P, dtype=torch.long)
    theta = positions.double()[a].t() * freq.double()          # [tokens][P]
    if inverse:
        theta = -theta
    i = 2 * torch.arange(P) if adjacent else torch.arange(P)
    j = i + 1 if adjacent else i + P
    u, v = x.double()[..., i], x.double()[..., j]
    cos, sin = torch.cos(theta)[:, None], torch.sin(theta)[:, None]
    y[..., i] = u * cos - v * sin
    y[..., j] = v * cos + u * sin
    return y


def check(got, x, want):
    # The turn's sine and cosine are off by a few half steps of fp32, products and sum by three more, of numbers as large as the pair at most:
    # 16 half steps of 2^-24 of twice the largest element; then the one rounding to bf16, half a step of 2^-8.
    got = got.double().cpu()
    tol = 2.0 ** -8 * want.abs() + 32 * 2.0 ** -24 * x.double().abs().max()
    assert torch.all((got - want).abs() <= tol), float(((got - want).abs() / tol).max())


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("tokens,hq,hkv,d,pairs,axes,far", [
    (1, 28, 4, 128, 64, 1, 40000), (33, 8, 2, 64, 32, 3, 500), (7, 1, 1, 16, 8, 2, 1 << 20), (100, 16, 1, 64, 24, 2, (1 << 31) - 200),
    (5, 6, 6, 256, 128, 4, 10), (3, 2, 1, 80, 40, 1, 3000), (513, 4, 4, 128, 16, 1, 99), (2, 40, 3, 72, 8, 1, 1)])
def test_against_the_definition(B, tokens, hq, hkv, d, pairs, axes, far, adjacent):
    gen = torch.Generator().manual_seed(tokens + d)
    q = torch.randn((tokens, hq, d), generator=gen).to(torch.bfloat16)
    k = torch.randn((tokens, hkv, d), generator=gen).to(torch.bfloat16)
    positions = torch.randint(0, far, (axes, tokens), generator=gen).to(torch.int32)
    positions[:, 0] = -positions[:, 0]
    freq = (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).to(torch.float32)
    axis = torch.randint(0, axes, (pairs,), generator=gen).to(torch.uint8) if axes > 1 else None
    r = B.Rotary(d, freq.to(DEV), axis.to(DEV) if axis is not None else None, axes, 1 if adjacent else 0)
    qd, kd, pd = q.to(DEV), k.to(DEV), positions.to(DEV)
    for inverse in (False, True):
        qo, ko = torch.full_like(qd, 7.0), torch.full_like(kd, 7.0)
        B.dynts_rotate(r, qd, kd, pd, qo, ko, inverse=inverse)
        check(qo, q, turn(q, positions, freq, axis, adjacent, inverse))
        check(ko, k, turn(k, positions, freq, axis, adjacent, inverse))
        assert torch.equal(qo[..., 2 * pairs:], qd[..., 2 * pairs:])
        alone = torch.full_like(qd, 7.0)
        B.dynts_rotate(r, qd, None, pd, alone, None, inverse=inverse)
        assert torch.equal(alone, qo)
        q2, k2 = qd.clone(), kd.clone()
        B.dynts_rotate(r, q2, k2, pd, q2, k2, inverse=inverse)  # in place
        assert torch.equal(q2, qo) and torch.equal(k2, ko)


@pytest.mark.parametrize("adjacent", [False, True])
def test_gradient(B, adjacent):
    """d/dx of sum(turn(x) * w) is the inverse turn of w: the definition's by autograd in float64, and by differences."""
    gen = torch.Generator().manual_seed(3)
    T, H, d, P, A = 9, 3, 64, 24, 2
    x = torch.randn((T, H, d), generator=gen).to(torch.bfloat16)
    w = torch.randn((T, H, d), generator=gen).to(torch.bfloat16)
    positions = torch.randint(0, 3000, (A, T), generator=gen).to(torch.int32)
    freq = torch.rand(P, generator=gen)
    axis = (torch.arange(P) % A).to(torch.uint8)
    leaf = x.double().requires_grad_()
    i = 2 * torch.arange(P) if adjacent else torch.arange(P)
    j = i + 1 if adjacent else i + P
    theta = positions.double()[axis.long()].t() * freq.double()
    u, v = leaf[..., i], leaf[..., j]
    y = leaf.clone().index_copy(2, i, u * torch.cos(theta)[:, None] - v * torch.sin(theta)[:, None])
    y = y.index_copy(2, j, v * torch.cos(theta)[:, None] + u * torch.sin(theta)[:, None])
    (y * w.double()).sum().backward()
    r = B.Rotary(d, freq.to(DEV), axis.to(DEV), A, 1 if adjacent else 0)
    got = torch.empty_like(w, device=DEV)
    B.dynts_rotate(r, w.to(DEV), None, positions.to(DEV), got, None, inverse=True)
    check(got, w, leaf.grad)
    f = lambda z: float((turn(z, positions, freq, axis, adjacent) * w.double()).sum())
    for at in [(0, 0, 0), (3, 1, 5), (8, 2, 47), (4, 0, 63)]:
        e = torch.zeros(x.shape, dtype=torch.float64)
        e[at] = 0.5
        slope = f(x.double() + e) - f(x.double() - e)   # (linear: differences of any size are exact up to float64)
        assert abs(float(got[at]) - slope) <= 2.0 ** -8 * abs(slope) + 32 * 2.0 ** -24 * float(w.abs().max())


def test_no_tokens(B):
    r = B.Rotary(64, torch.ones(32, device=DEV))
    e = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    B.dynts_rotate(r, e, None, torch.empty((1, 0), dtype=torch.int32, device=DEV), e, None)
