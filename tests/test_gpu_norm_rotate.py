"""Head norms, position rotation and the append to pages against their definition in 64 bits."""
import pytest
import torch

import paper_2502_11494_amd as D

import attend_util as A

pytestmark = pytest.mark.gpu

EPS = 1e-6


def definition(x, heads, d, rot, pos, sections, inv_freq, interleaved, weight, scale):
    """[T, heads, d] in 64 bits, and how far the 32-bit arithmetic before the last rounding may be off."""
    T = x.shape[0]
    x = x.double().reshape(T, heads, d)
    u, size = 2.0 ** -24, x.abs()
    err = torch.zeros_like(x)
    if weight is not None:
        r = 1 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
        x = x * r * weight.double()
        # the mean: d terms; its root's reciprocal halves a relative error; the function; two products
        size, err = x.abs(), x.abs() * (d / 2 + 8) * u
    half = rot // 2
    plane = [p for p, m in enumerate(sections) for _ in range(m)]
    theta = torch.stack([pos[p].double() for p in plane], 1) * inv_freq.double() if half else torch.zeros((T, 0)).double()
    a = slice(0, rot, 2) if interleaved else slice(0, half)
    b = slice(1, rot, 2) if interleaved else slice(half, rot)
    y, tol = x.clone(), err.clone()
    c, s = theta.cos()[:, None] * scale, theta.sin()[:, None] * scale
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    both = (size[..., a] + size[..., b]) * abs(scale)
    # the angle's sine and cosine to 8 units, their scaling, the products and the sum
    tol[..., a] = tol[..., b] = (err[..., a] + err[..., b]) * abs(scale) + 14 * u * both
    return y, tol


def inputs(T, Hq, Hkv, d, rot, planes, dtype, norm, seed=0, far=0):
    g = torch.Generator().manual_seed(seed)
    t = A.TYPES[dtype]
    rows = torch.full((T, (Hq + 2 * Hkv) * d + 16), float("nan"), dtype=t)
    rows[:, :-16] = torch.randn((T, (Hq + 2 * Hkv) * d), generator=g).to(t)
    pos = torch.randint(0, 16384, (planes, T), generator=g) + far
    half = rot // 2
    inv_freq = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float()
    sections = [half] if planes == 1 else [half // 4, half // 2 - half // 4] + [half - half // 2] if planes == 3 else [1, 0, 0, half - 1]
    w = lambda: (torch.randn(d, generator=g) + 1.5).to(t) if norm else None  # noqa: E731
    return rows, pos, inv_freq, sections, w(), w()


def gpu(x):
    return None if x is None else x.cuda()


def within(got, want, tol, dtype):
    err = (got.double() - want).abs()
    allowed = 1.01 * (tol + A.UNIT[dtype] * (want.abs() + tol)) + 1e-37
    assert torch.isfinite(got.float()).all()
    assert bool((err <= allowed).all()), f"{float((err / allowed).max()):.3g} times what the arithmetic allows"


SHAPES = [(4, 4, 128, 128), (28, 4, 128, 128), (7, 1, 128, 64), (6, 2, 64, 64), (3, 3, 80, 80), (4, 2, 80, 40), (2, 2, 96, 48),
          (9, 3, 256, 256), (2, 1, 256, 64), (5, 5, 8, 8), (4, 4, 72, 24), (3, 1, 64, 0), (33, 11, 40, 32)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,rot", SHAPES)
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rows(dtype, Hq, Hkv, d, rot, norm, interleaved):
    for T, planes, scale in ((1, 1, 1.0), (37, 3, 1.25), (4099, 1, 1.0)):
        if rot < 16:
            planes = 1
        rows, pos, inv_freq, sections, qw, kw = inputs(T, Hq, Hkv, d, rot, planes, dtype, norm, seed=T + d)
        x = rows.cuda()
        q, k = x[:, :Hq * d], x[:, Hq * d:(Hq + Hkv) * d]
        r = D.make_rotation(Hq, Hkv, d, A.KIND[rows.dtype], inv_freq.cuda(), interleaved=interleaved, sections=sections,
                            q_weight=gpu(qw), k_weight=gpu(kw), eps=EPS, scale=scale)
        qo = torch.full((T, Hq * d + 8), 5.0, dtype=rows.dtype, device="cuda")
        ko = torch.full((T, Hkv * d), 5.0, dtype=rows.dtype, device="cuda")
        l1 = torch.empty(T, device="cuda")
        D.dart_norm_rotate(r, q, k, pos.cuda() if planes > 1 else pos[0].cuda(), qo[:, :Hq * d], ko, l1_out=l1)
        torch.cuda.synchronize()
        assert bool((qo[:, Hq * d:] == 5.0).all())
        for got, src, heads, w in ((qo[:, :Hq * d], q, Hq, qw), (ko, k, Hkv, kw)):
            want, tol = definition(src.cpu(), heads, d, rot, pos, sections, inv_freq, interleaved, w, scale)
            within(got.cpu().view(T, heads, d), want, tol, rows.dtype)
        exact = ko.cpu().double().abs().sum(1)
        assert bool(((l1.cpu().double() - exact).abs() <= 2.0 ** -20 * exact).all())


def test_in_place_and_one_norm_of_two():
    rows, pos, inv_freq, sections, qw, kw = inputs(50, 4, 2, 64, 64, 1, "bf16", True, seed=1)
    for weights in (dict(q_weight=qw.cuda()), dict(k_weight=kw.cuda())):
        x = rows.cuda()
        q, k = x[:, :256], x[:, 256:384]
        r = D.make_rotation(4, 2, 64, D.DART_BF16, inv_freq.cuda(), **weights)
        apart = torch.empty((50, 256), dtype=rows.dtype, device="cuda"), torch.empty((50, 128), dtype=rows.dtype, device="cuda")
        D.dart_norm_rotate(r, q, k, pos[0].cuda(), *apart)
        D.dart_norm_rotate(r, q, k, pos[0].cuda(), q, k)
        torch.cuda.synchronize()
        assert torch.equal(q, apart[0]) and torch.equal(k, apart[1])
        assert torch.equal(x[:, 384:512].cpu(), rows[:, 384:512]), "what lies beside the rows is left alone"
        want, tol = definition(rows[:, 256:384], 2, 64, 64, pos, sections, inv_freq, False,
                               kw if "k_weight" in weights else None, 1.0)
        within(k.cpu().view(50, 2, 64), want, tol, rows.dtype)


@pytest.mark.parametrize("far", [0, 10 ** 6, 2 ** 31 + 12345, -(10 ** 5)])
def test_positions_of_any_size_keep_their_angles(far):
    rows, pos, inv_freq, sections, _, _ = inputs(20, 2, 2, 128, 128, 1, "f32", False, seed=2, far=far)
    q, k = rows[:, :256].cuda(), rows[:, 256:512].cuda()
    r = D.make_rotation(2, 2, 128, D.DART_F32, inv_freq.cuda())
    qo, ko = torch.empty((20, 256), device="cuda"), torch.empty((20, 256), device="cuda")
    D.dart_norm_rotate(r, q, k, pos[0].cuda(), qo, ko)
    torch.cuda.synchronize()
    want, tol = definition(rows[:, :256], 2, 128, 128, pos, sections, inv_freq, False, None, 1.0)
    within(qo.cpu().view(20, 2, 128), want, tol, torch.float32)


def test_position_zero_changes_nothing_and_turns_keep_lengths():
    rows, pos, inv_freq, _, _, _ = inputs(30, 2, 1, 64, 64, 1, "f32", False, seed=3)
    q, k = rows[:, :128].cuda(), rows[:, 128:192].cuda()
    r = D.make_rotation(2, 1, 64, D.DART_F32, inv_freq.cuda())
    qo, ko = torch.empty((30, 128), device="cuda"), torch.empty((30, 64), device="cuda")
    D.dart_norm_rotate(r, q, k, torch.zeros(30, dtype=torch.int64, device="cuda"), qo, ko)
    assert torch.equal(qo, q) and torch.equal(ko, k)
    D.dart_norm_rotate(r, q, k, pos[0].cuda(), qo, ko)
    a, b = qo.view(30, 2, 64).double().norm(dim=-1), q.reshape(30, 2, 64).double().norm(dim=-1)
    assert bool(((a - b).abs() <= 1e-6 * b).all())


def test_a_row_that_is_no_number_stays_alone():
    rows, pos, inv_freq, _, qw, kw = inputs(9, 4, 2, 64, 64, 1, "bf16", True, seed=4)
    r = D.make_rotation(4, 2, 64, D.DART_BF16, inv_freq.cuda(), q_weight=qw.cuda(), k_weight=kw.cuda())

    def run(x):
        x = x.cuda()
        qo = torch.empty((9, 256), dtype=x.dtype, device="cuda")
        ko = torch.empty((9, 128), dtype=x.dtype, device="cuda")
        D.dart_norm_rotate(r, x[:, :256], x[:, 256:384], pos[0].cuda(), qo, ko)
        return qo.cpu().view(9, 4, 64), ko.cpu().view(9, 2, 64)

    clean = run(rows)
    bad = rows.clone()
    bad[3, 64:128] = float("nan")
    bad[5, 256 + 70] = float("inf")
    q, k = run(bad)
    assert torch.isnan(q[3, 1]).all()
    q[3, 1], k[5, 1] = clean[0][3, 1], clean[1][5, 1]
    assert torch.equal(q, clean[0]) and torch.equal(k, clean[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["heads", "rows"])
@pytest.mark.parametrize("Hq,Hkv,d,page", [(4, 4, 128, 16), (28, 4, 128, 64), (6, 2, 80, 1), (4, 1, 256, 32)])
def test_append(dtype, order, Hq, Hkv, d, page):
    n = [1, 0, 5, 17, 40, 1, 64]
    kv = [30, 12, 5, 50, 140, 1, 64]
    for one_each in (False, True):
        if one_each:
            n = [1] * 7
        c = A.make(n, kv, Hq, Hkv, d, page, dtype, order, seed=page)
        T = c.T
        rows, pos, inv_freq, sections, qw, kw = inputs(T, Hq, Hkv, d, d, 3, dtype, True, seed=5)
        x = rows.cuda()
        q, k, v = x[:, :Hq * d], x[:, Hq * d:(Hq + Hkv) * d], x[:, (Hq + Hkv) * d:(Hq + 2 * Hkv) * d]
        r = D.make_rotation(Hq, Hkv, d, A.KIND[c.dtype], inv_freq.cuda(), sections=sections, q_weight=qw.cuda(),
                            k_weight=kw.cuda(), eps=EPS)
        kp, vp = A.pool_to_gpu(c.k_pool, order), A.pool_to_gpu(c.v_pool, order)
        cache = A.cache_of(c, kp)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        qo = torch.empty((T, Hq * d), dtype=c.dtype, device="cuda")
        ko = torch.empty((T, Hkv * d), dtype=c.dtype, device="cuda")
        l1 = torch.empty(T, device="cuda")
        D.dart_norm_rotate_append(r, cache, q, k, v, pos.cuda(), qo, kp, vp, k_out=ko, l1_out=l1, status=status)
        torch.cuda.synchronize()
        assert int(status) == 0
        want, tol = definition(k.cpu(), Hkv, d, d, pos, sections, inv_freq, False, kw, 1.0)
        within(ko.cpu().view(T, Hkv, d), want, tol, c.dtype)
        want, tol = definition(q.cpu(), Hq, d, d, pos, sections, inv_freq, False, qw, 1.0)
        within(qo.cpu().view(T, Hq, d), want, tol, c.dtype)
        # the pages hold the same key rows, the values as they came, and what they held elsewhere
        for pool, was, new in ((kp, c.k_pool, ko.cpu()), (vp, c.v_pool, v.cpu())):
            expect = was.clone()
            for b in range(len(n)):
                w = torch.arange(kv[b] - n[b], kv[b])
                expect[c.table[b].long()[w // page], :, w % page] = new[int(c.cu[b]):int(c.cu[b + 1])].reshape(-1, Hkv, d)
            same = (pool.cpu() == expect) | (torch.isnan(pool.cpu()) & torch.isnan(expect))
            assert bool(same.all())
        exact = ko.cpu().double().abs().sum(1)
        assert bool(((l1.cpu().double() - exact).abs() <= 2.0 ** -20 * exact).all())
        before = kp.clone()
        D.dart_norm_rotate_append(r, cache, q, k, v, pos.cuda(), qo, kp, vp)  # (without the optional outputs)
        assert torch.equal(torch.nan_to_num(before), torch.nan_to_num(kp))


def test_tokens_that_have_no_place_are_flagged_and_left_out():
    n, kv = [2, 3, 4], [10, 20, 30]
    c = A.make(n, kv, 4, 2, 64, 16, "bf16", seed=6)
    rows, pos, inv_freq, sections, _, _ = inputs(9, 4, 2, 64, 64, 1, "bf16", False, seed=6)
    x = rows.cuda()
    q, k, v = x[:, :256], x[:, 256:384], x[:, 384:512]
    r = D.make_rotation(4, 2, 64, D.DART_BF16, inv_freq.cuda())
    qo = torch.empty((9, 256), dtype=c.dtype, device="cuda")
    good = c.k_pool.cuda(), c.v_pool.cuda()
    D.dart_norm_rotate_append(r, A.cache_of(c, good[0]), q, k, v, pos[0].cuda(), qo, *good)
    q_good = qo.clone()

    def left_out(b, bit, **how):
        kp, vp = c.k_pool.cuda(), c.v_pool.cuda()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        qo.zero_()
        D.dart_norm_rotate_append(r, A.cache_of(c, kp, **how), q, k, v, pos[0].cuda(), qo, kp, vp, status=status)
        torch.cuda.synchronize()
        assert int(status) == bit and torch.equal(qo, q_good)
        for got, full, was in ((kp, good[0], c.k_pool), (vp, good[1], c.v_pool)):
            expect = full.cpu().clone()
            w = torch.arange(kv[b] - n[b], kv[b])
            p, i = c.table[b].long()[w // 16], w % 16
            expect[p, :, i] = was[p, :, i]
            assert torch.equal(torch.nan_to_num(got.cpu()), torch.nan_to_num(expect))

    left_out(1, 1, kv=torch.tensor([10, 2, 30], dtype=torch.int32))     # fewer keys than tokens
    left_out(1, 1, kv=torch.tensor([10, 2000, 30], dtype=torch.int32))
    left_out(1, 1, kv=torch.tensor([10, -20, 30], dtype=torch.int32))
    left_out(2, 1, max_q=3)
    table = c.table.clone()
    table[1, 1] = c.k_pool.shape[0]
    left_out(1, 2, table=table)
    # offsets that are none: memory-safe, flagged
    kp, vp = c.k_pool.cuda(), c.v_pool.cuda()
    for cu in ([0, 5, 2, 9], [4, 5, 6, 9], [-3, 2, 5, 9], [0, 2, 5, 99]):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        D.dart_norm_rotate_append(r, A.cache_of(c, kp, cu=torch.tensor(cu, dtype=torch.int32)), q, k, v, pos[0].cuda(), qo, kp, vp,
                                  status=status)
        torch.cuda.synchronize()
        assert int(status) == 1 and torch.equal(qo, q_good)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,page", [(4, 2, 64, 16), (28, 4, 128, 64), (16, 16, 128, 1), (3, 1, 40, 8)])
def test_append_of_many_tokens(dtype, Hq, Hkv, d, page):
    """A wave to a token, or four with several rounds of heads each: pages hold what the call without pages gives."""
    n, kv = [700, 1, 0, 613], [1000, 1, 9, 613]
    c = A.make(n, kv, Hq, Hkv, d, page, dtype, seed=page + d)
    T = c.T
    rows, pos, inv_freq, sections, qw, kw = inputs(T, Hq, Hkv, d, d, 3, dtype, True, seed=7)
    x = rows.cuda()
    q, k, v = x[:, :Hq * d], x[:, Hq * d:(Hq + Hkv) * d], x[:, (Hq + Hkv) * d:(Hq + 2 * Hkv) * d]
    r = D.make_rotation(Hq, Hkv, d, A.KIND[c.dtype], inv_freq.cuda(), sections=sections, q_weight=qw.cuda(),
                        k_weight=kw.cuda(), eps=EPS)
    qo, q1 = (torch.empty((T, Hq * d), dtype=c.dtype, device="cuda") for _ in range(2))
    k1 = torch.empty((T, Hkv * d), dtype=c.dtype, device="cuda")
    kp, vp = A.pool_to_gpu(c.k_pool, "heads"), A.pool_to_gpu(c.v_pool, "heads")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    D.dart_norm_rotate(r, q, k, pos.cuda(), q1, k1)
    D.dart_norm_rotate_append(r, A.cache_of(c, kp), q, k, v, pos.cuda(), qo, kp, vp, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and torch.equal(qo, q1)
    for got, heads, w in ((q1, Hq, qw), (k1, Hkv, kw)):
        src = q if got is q1 else k
        want, tol = definition(src.cpu(), heads, d, d, pos, sections, inv_freq, False, w, 1.0)
        within(got.cpu().view(T, heads, d), want, tol, c.dtype)
    for pool, was, new in ((kp, c.k_pool, k1.cpu()), (vp, c.v_pool, v.cpu())):
        expect = was.clone()
        for b in range(len(n)):
            w = torch.arange(kv[b] - n[b], kv[b])
            expect[c.table[b].long()[w // page], :, w % page] = new[int(c.cu[b]):int(c.cu[b + 1])].reshape(-1, Hkv, d)
        same = (pool.cpu() == expect) | (torch.isnan(pool.cpu()) & torch.isnan(expect))
        assert bool(same.all())
