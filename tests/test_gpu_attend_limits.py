"""Attention and rotation at the sizes that the header names as the largest."""
import pytest
import torch

import paper_2502_11494_amd as D

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("packed", [False, True])
def test_a_token_for_each_of_the_most_sequences(packed):
    """2^20 sequences of eight key heads: more blocks than one launch takes."""
    B, H, d, page, n_pages = 1 << 20, 8, 8, 4, 97
    g = torch.Generator(device="cuda").manual_seed(1)
    k_pool, v_pool = (torch.randn((n_pages, H, page, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((B, H * d), generator=g, device="cuda").bfloat16()
    b = torch.arange(B, device="cuda")
    table, kv = (b % n_pages).int().view(B, 1), (b % (page + 1)).int()
    cu = torch.arange(B + 1, dtype=torch.int32, device="cuda") if packed else None
    cache = D.make_cache(H, k_pool, table, kv, page, T=B, max_q=1, cu_q=cu)
    out, lse = torch.full_like(q, 7.0), torch.full((B, H), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    D.dart_attend(cache, q, k_pool, v_pool, out, D.alloc_attend_workspace(cache), scale=0.5, lse=lse, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    u = 2.0 ** -24
    for at in range(0, B, 1 << 17):
        x = slice(at, at + (1 << 17))
        k, v = (p.double()[table[x, 0].long()] for p in (k_pool, v_pool))  # [n, H, page, d]
        qq = q[x].double().view(-1, H, 1, d)
        seen = (torch.arange(page, device="cuda") < kv[x, None])[:, None].expand(-1, H, -1)
        s = ((qq * k).sum(-1) * 0.5).masked_fill(~seen, -float("inf"))
        some = seen.any(-1)
        m = torch.where(some, s.amax(-1), 0.0)
        p = torch.exp(s - m[..., None])
        l = torch.where(some, p.sum(-1), 1.0)
        y = torch.where(some[..., None], (p[..., None] * v).sum(2) / l[..., None], 0.0)
        size = (p[..., None] * v.abs()).sum(2) / l[..., None]
        # a score's error is its weight's; the weights' and the result's rounding
        e = (d + 4) * u * (qq.abs() * k.abs()).sum(-1).amax(-1) * 0.5 + 8 * u * (1 + m.abs())
        tol = 1.01 * ((2 * e[..., None] + 2.0 ** -8 + 140 * u) * size + 2.0 ** -8 * y.abs()) + 1e-37
        assert bool(((out[x].double().view(-1, H, d) - y).abs() <= tol).all()), at
        want = torch.where(some, m + torch.log(l), -float("inf"))
        assert torch.equal(lse[x] == -float("inf"), ~some)
        off = (lse[x].double() - want).abs()[some]
        assert bool((off <= 1.01 * (e[some] + 140 * u + 8 * u * (1 + want[some].abs()))).all()), at


def test_rotation_of_the_most_tokens():
    """2^24 tokens of rows long enough that four waves would share one: in place, 73 GB."""
    T, Hq, d, rot = 1 << 24, 15, 136, 8
    width, period = (Hq + 1) * d, 1024
    if torch.cuda.mem_get_info()[0] < 2 * T * width + (20 << 30):
        pytest.skip("needs 93 GB of free memory")
    g = torch.Generator(device="cuda").manual_seed(2)
    base = torch.randn((period, width), generator=g, device="cuda").bfloat16()
    pos = torch.arange(period, device="cuda")
    r = D.make_rotation(Hq, 1, d, D.DART_BF16, torch.tensor([1.0, 0.3, 0.1, 0.01], device="cuda"))
    few = base.clone()
    D.dart_norm_rotate(r, few[:, :Hq * d], few[:, Hq * d:], pos, few[:, :Hq * d], few[:, Hq * d:])
    x = torch.empty((T, width), dtype=torch.bfloat16, device="cuda")
    x.view(-1, period, width).copy_(base.expand(T // period, -1, -1))
    l1 = torch.zeros(T, device="cuda")
    D.dart_norm_rotate(r, x[:, :Hq * d], x[:, Hq * d:], pos.repeat(T // period), x[:, :Hq * d], x[:, Hq * d:], l1_out=l1)
    torch.cuda.synchronize()
    assert not torch.equal(few, base)
    for part in x.view(-1, period, width).split(512):
        assert bool((part == few).all())
    assert bool((l1.view(-1, period) == l1[:period]).all())
    assert bool(((l1[:period].double() - few[:, Hq * d:].double().abs().sum(1)).abs() <= 2.0 ** -20 * l1[:period]).all())
    del x, part
    torch.cuda.empty_cache()
