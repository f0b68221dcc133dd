"""Attention where scores are large: weights, sums and logarithms have to hold wherever the scores do."""
import pytest
import torch

import paper_2502_11494_amd as D

import attend_util as A

pytestmark = pytest.mark.gpu

STEPS = (1.0, 1.25, 1.5, 1.75)


def spiked(n, kv, Hq, Hkv, d, dtype, query, key, seed, idle=False, **more):
    """Queries and keys of one element each, query * key * (1, 1.25, 1.5 or 1.75): scores are exact products, and any two of a row
    are the same or far apart.  The element's place differs from head to head.  idle: the queries of every other token are
    zeros, and so are its scores."""
    c = A.make(n, kv, Hq, Hkv, d, 16, dtype, seed=seed, **more)
    g = torch.Generator().manual_seed(seed + 1)
    r = Hq // Hkv
    place = torch.arange(Hkv) * 5 % d
    k = torch.zeros_like(c.k_pool)
    steps = torch.tensor(STEPS)[torch.randint(0, 4, c.k_pool.shape[:3], generator=g)] * key
    for h in range(Hkv):
        k[:, h, :, place[h]] = steps[:, h].to(c.dtype)
    c.k_pool = torch.where(torch.isnan(c.k_pool), c.k_pool, k)  # (rows of nobody stay NaN)
    q = torch.zeros((c.T, Hq, d), dtype=c.dtype)
    for j in range(Hq):
        q[:, j, place[j // r]] = query
    if idle:
        q[1::2] = 0
    c.q = q.view(c.T, Hq * d)
    return c


def definition(c, scale, causal):
    """In 64 bits.  The weights are those of the largest scores, all alike; what the arithmetic may be off by: the sums, the
    weights' rounding for bf16 rows, the result's; of the logarithm the products that make the score."""
    r = c.Hq // c.Hkv
    out, lse = torch.zeros((c.T, c.Hq, c.d), dtype=torch.float64), torch.full((c.T, c.Hq), -float("inf"), dtype=torch.float64)
    tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    u = 2.0 ** -24
    group = [g for g, m in enumerate(c.group_of or []) for _ in range(m)]
    q = c.q.double().view(c.T, c.Hq, c.d)
    for b, (n, kv) in enumerate(zip(c.n, c.kv)):
        front = c.prefix[group[b]] if group else 0
        for i in range(n):
            t, own = int(c.cu[b]) + i, min(kv, kv - n + i + 1) if causal else kv
            for h in range(c.Hkv):
                k, v = A.keys_of(c, c.k_pool, c.table[b], own, h), A.keys_of(c, c.v_pool, c.table[b], own, h)
                if front:
                    k = torch.cat((A.keys_of(c, c.k_pool, c.front[group[b]], front, h), k))
                    v = torch.cat((A.keys_of(c, c.v_pool, c.front[group[b]], front, h), v))
                s = (q[t, h * r:(h + 1) * r] @ k.T) * torch.tensor(scale, dtype=torch.float32).double()
                m = s.amax(1, keepdim=True)
                p = torch.exp(s - m)
                near = s[(s < m)]
                assert near.numel() == 0 or float((m - s)[s < m].min()) > 200
                y, size, total = p @ v / p.sum(1, keepdim=True), p @ v.abs() / p.sum(1, keepdim=True), own + front + 64
                w = A.UNIT[torch.bfloat16] if c.dtype == torch.bfloat16 else 0.0
                out[t, h * r:(h + 1) * r], lse[t, h * r:(h + 1) * r] = y, m[:, 0] + torch.log(p.sum(1))
                tol[t, h * r:(h + 1) * r] = 1.01 * ((w + 2 * total * u) * size + A.UNIT[c.dtype] * y.abs()) + 1e-37
                lse_tol[t, h * r:(h + 1) * r] = 1.01 * (2 * total * u + 8 * u * (1 + m[:, 0].abs() + torch.log(p.sum(1))))
    return out, lse, tol, lse_tol


def check(c, scale, causal=True, **how):
    out, lse = A.attend(c, scale=scale, causal=causal, **how)
    want, want_lse, tol, lse_tol = definition(c, scale, causal)
    assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
    err, off = (out.double() - want).abs(), (lse.double() - want_lse).abs()
    assert bool((err <= tol).all()), f"out: {float((err / tol).max()):.3g} times what the arithmetic allows"
    assert bool((off <= lse_tol).all()), f"lse: {float((off / lse_tol).max()):.3g} times what the arithmetic allows"


MAGNITUDES = [(1e3, 1e3), (1e6, 1e6), (1e5, -1e6), (3e9, 1e9), (-1e12, 1e12), (1e18, 1e18), (1e25, 1e12)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("query,key", MAGNITUDES)
def test_large_scores(dtype, query, key):
    for scale in (0.0884, 1.0):
        # a few rows, four waves of rows, heads of every width, a long context in parts
        check(spiked([1, 3], [131, 40], 4, 2, 128, dtype, query, key, 1), scale)
        check(spiked([70, 33], [90, 300], 4, 4, 64, dtype, query, key, 2), scale)
        check(spiked([1, 9], [30, 20], 7, 1, 256, dtype, query, key, 3), scale, causal=False)
        check(spiked([1], [5000], 6, 2, 80, dtype, query, key, 4), scale)
        check(spiked([5, 40], [300, 77], 4, 2, 64, dtype, query, key, 7, idle=True), scale)
        check(spiked([1, 2, 1], [5, 70, 1], 4, 2, 64, dtype, query, key, 5, groups=[2, 1], prefix=[300, 33]), scale)


def test_one_key_is_its_value_whatever_its_score():
    for dtype in ("bf16", "f32"):
        for query, key in MAGNITUDES:
            c = spiked([1, 1], [1, 1], 4, 2, 64, dtype, query, key, 6)
            out, _ = A.attend(c, scale=0.7)
            for b in range(2):
                v = torch.stack([A.keys_of(c, c.v_pool, c.table[b], 1, h)[0] for h in (0, 0, 1, 1)])
                assert torch.equal(out[b].double(), v)


def test_large_scores_in_the_widest_tiles():
    """One head's scores are large, the others' are not."""
    n = [300, 257, 64, 129, 512, 31, 255, 400, 256, 200, 333, 65, 128, 300, 450, 290, 256, 260]
    c = A.make(n, n, 32, 32, 64, 64, "bf16", seed=5)
    assert sum(n) // 256 * 32 >= 384 and max(n) > 128
    c.q = c.q.clone()
    q = c.q.view(c.T, 32, 64)
    want, want_lse, tol, lse_tol = A.reference(c, 0.125, True)
    spike = c.k_pool[:, 7].clone()
    g = torch.Generator().manual_seed(6)
    spike = torch.where(torch.isnan(spike), spike, torch.zeros_like(spike))
    spike[..., 3] = torch.where(torch.isnan(spike[..., 3]), spike[..., 3],
                                (torch.tensor(STEPS)[torch.randint(0, 4, spike.shape[:2], generator=g)] * 2.0 ** 40).bfloat16())
    c.k_pool[:, 7] = spike
    q[:, 7] = 0
    q[:, 7, 3] = 2.0 ** 30
    out, lse = A.attend(c, scale=0.125, max_kv=5000)
    others = [h for h in range(32) if h != 7]
    assert bool(((out.double() - want).abs() <= tol)[:, others].all())
    assert bool(((lse.double() - want_lse).abs() <= lse_tol)[:, others].all())
    for b, m in enumerate(n):
        k, v = A.keys_of(c, c.k_pool, c.table[b], m, 7)[:, 3], A.keys_of(c, c.v_pool, c.table[b], m, 7)
        seen = torch.ones((m, m), dtype=torch.bool).tril()
        top = torch.where(seen, k[None], 0.0).amax(1, keepdim=True)
        p = ((k[None] == top) & seen).double()
        y, size = p @ v / p.sum(1, keepdim=True), p @ v.abs() / p.sum(1, keepdim=True)
        got = out[int(c.cu[b]):int(c.cu[b + 1]), 7].double()
        assert bool(((got - y).abs() <= 1.01 * ((2.0 ** -8 + 2 * (m + 64) * 2.0 ** -24) * size + 2.0 ** -8 * y.abs()) + 1e-37).all())
