"""Sines and cosines of the rotation themselves, where they are small: the angle is held in 64 bits all the way."""
import pytest
import torch

import paper_2502_11494_amd as D

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1.0, -2.0])
def test_small_sines_and_cosines_keep_their_digits(scale):
    T, half = 4096, 128
    g = torch.Generator().manual_seed(1)
    pos = torch.arange(T) - T // 2
    inv_freq = torch.rand(half, generator=g) * 0.9 + 0.1
    inv_freq[0] = 1.0
    theta = pos.double()[:, None] * inv_freq.double()
    x = torch.zeros((T, 2 * half))
    x[:, :half] = 1.0  # (1, 0) becomes (cos, sin)
    r = D.make_rotation(1, 1, 2 * half, D.DART_F32, inv_freq.cuda(), scale=scale)
    q, k = torch.empty((T, 2 * half), device="cuda"), torch.empty((T, 2 * half), device="cuda")
    D.dart_norm_rotate(r, x.cuda(), x.cuda(), pos.cuda(), q, k)
    torch.cuda.synchronize()
    want = torch.cat((theta.cos(), theta.sin()), 1) * scale
    # of the value: the function (4 units), its correction, scaling; of the angle: two 64-bit products of up to 2000
    allowed = (8 * 2.0 ** -24) * want.abs() + abs(scale) * 4 * theta.abs().amax() * 2.0 ** -53
    small = want.abs() < 1e-3 * abs(scale)
    assert int(small.sum()) > 300
    for got in (q, k):
        err = (got.cpu().double() - want).abs()
        assert bool((err <= allowed).all()), f"{float((err / allowed).max()):.3g} times what the arithmetic allows"
