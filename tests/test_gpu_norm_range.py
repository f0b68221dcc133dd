"""Head norms of rows whose squares leave the range of 32 bits, against the definition in 64."""
import pytest
import torch

import paper_2502_11494_amd as D

import attend_util as A

pytestmark = pytest.mark.gpu

LARGEST = 3.3e38


def rows_of(T, heads, d, factors, dtype, g):
    """[T, heads, d]: every head of a magnitude of its own, all elements within a factor of four of it."""
    x = (torch.rand((T, heads, d), generator=g) * 0.75 + 0.25) * (torch.randint(0, 2, (T, heads, d), generator=g) * 2 - 1)
    f = torch.tensor(factors, dtype=torch.float64)[torch.randint(0, len(factors), (T, heads, 1), generator=g)]
    return (x.double() * f).to(A.TYPES[dtype])


def normed(x, weight, eps):
    """In 64 bits, and what 32-bit arithmetic may be off by before the last rounding: the mean of d terms (its root's
    reciprocal halves a relative error), the function, the scaling of eps, two products."""
    x = x.double()
    y = x / (x.square().mean(-1, keepdim=True) + torch.tensor(eps, dtype=torch.float32).double()).sqrt()
    if weight is not None:
        y = y * weight.double()
    return y, (x.shape[-1] / 2 + 8) * 2.0 ** -24 * y.abs()


def close(got, want, tol, dtype):
    allowed = 1.01 * (tol + A.UNIT[dtype] * (want.abs() + tol)) + 2.0 ** -133  # (the spacing of the least bf16 numbers)
    err = (got.double() - want).abs()
    assert torch.isfinite(got.float()).all()
    assert bool((err <= allowed).all()), f"{float((err / allowed).max()):.3g} times what the arithmetic allows"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 128), (28, 4, 128), (3, 3, 8), (6, 2, 80), (4, 2, 256), (9, 9, 40)])
@pytest.mark.parametrize("factors,eps", [
    ([1e25], 1e-6), ([LARGEST], 1e-6), ([LARGEST, 1.0, 1e20], 0.0), ([1e-25], 0.0), ([1e-39, 1e-25, 1.0], 0.0),
    ([1e-25, 1e30], 1e-6), ([1e-15, 1e-16, 1e-14], 1e-30), ([1e-25, 1e-18], 1e-40), ([1e19, 2e19, 5e18], 0.0), ([1.0], 1e38)])
def test_heads_of_any_magnitude(dtype, Hq, Hkv, d, factors, eps):
    g = torch.Generator().manual_seed(d)
    inv_freq = torch.ones(0, device="cuda")
    for T in (1, 33, 1100):  # (four waves to a token, one)
        q, k = rows_of(T, Hq, d, factors, dtype, g), rows_of(T, Hkv, d, factors, dtype, g)
        qw, kw = ((torch.rand(d, generator=g) + 0.5).to(q.dtype) for _ in range(2))
        r = D.make_rotation(Hq, Hkv, d, A.KIND[q.dtype], inv_freq, q_weight=qw.cuda(), k_weight=kw.cuda(), eps=eps)
        qo, ko = (torch.empty((T, h * d), dtype=q.dtype, device="cuda") for h in (Hq, Hkv))
        l1 = torch.empty(T, device="cuda")
        D.dart_norm_rotate(r, q.cuda(), k.cuda(), torch.zeros(T, dtype=torch.int64, device="cuda"), qo, ko, l1_out=l1)
        torch.cuda.synchronize()
        for got, x, w in ((qo, q, qw), (ko, k, kw)):
            close(got.cpu().view(x.shape), *normed(x, w, eps), q.dtype)
        exact = ko.cpu().double().abs().sum(1)
        assert bool(((l1.cpu().double() - exact).abs() <= 2.0 ** -20 * exact + 2.0 ** -140).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_weight_keep_their_magnitude(dtype):
    """Only the queries are normed: the keys beside them pass, bit for bit, and rotated pairs keep their length."""
    g = torch.Generator().manual_seed(5)
    q, k = rows_of(40, 4, 64, [1e25, 1e-25], dtype, g), rows_of(40, 2, 64, [1e25, 1e-25], dtype, g)
    w = torch.ones(64, dtype=q.dtype)
    r = D.make_rotation(4, 2, 64, A.KIND[q.dtype], torch.ones(32, device="cuda"), q_weight=w.cuda(), eps=0.0)
    qo, ko = (torch.empty((40, h * 64), dtype=q.dtype, device="cuda") for h in (4, 2))
    D.dart_norm_rotate(r, q.cuda(), k.cuda(), torch.zeros(40, dtype=torch.int64, device="cuda"), qo, ko)
    torch.cuda.synchronize()
    assert torch.equal(ko.cpu().view(k.shape), k)
    close(qo.cpu().view(q.shape), *normed(q, w, 0.0), q.dtype)
