"""Caches held in 4 bits on the GPU: rows to pages and back, bit for bit by the format's definition, and attention over them
against its definition in 64 bits over the values that the codes stand for (attend_util.reference)."""
import pytest
import torch

import attend_util as A
import more_gpu as G
import more_util as U
import paper_2502_11494_amd as D

pytestmark = pytest.mark.gpu

RAGGED_N = [1, 0, 3, 17, 1, 64, 33, 5, 1, 130]
RAGGED_KV = [1, 9, 3, 40, 0, 65, 20, 128, 300, 257]


def wild(T, width, dtype, seed):
    """Rows of blocks of every magnitude, with values on the borders between codes, zeros of both signs and odd blocks."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, width), generator=g)
    x *= torch.exp2(torch.randint(-120, 120, (T, width // 8), generator=g).float()).repeat_interleave(8, 1)[:, :width] if seed % 2 else 1.0
    grid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 6.98, 0.0, -0.0])
    some = torch.rand((T, width), generator=g) < 0.3
    x[some] = grid[torch.randint(0, len(grid), (int(some.sum()),), generator=g)] * (1 - 2 * torch.randint(0, 2, (int(some.sum()),), generator=g))
    return x.to(dtype)


def check_append(c, got, k, v):
    before = c.four
    for have, old, x in zip(got[:2], before, (k, v)):
        want = tuple(t.clone() for t in old)
        packed = U.pack(x.reshape(c.T, -1, c.d))
        for b, n in enumerate(c.n):
            if n == 0 or c.kv[b] < n:
                continue
            page, row = (t[-n:] for t in U.places(c, b))
            for w, p in zip(want, packed):
                w[page, :, row] = p[int(c.cu[b]):int(c.cu[b + 1])]
        for a, w in zip(have, want):  # (rows of no token are left alone)
            assert torch.equal(a, w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv,d,order", [(4, 128, "heads"), (1, 8, "heads"), (3, 40, "rows"), (2, 80, "heads"), (2, 96, "rows"),
                                         (5, 64, "heads"), (2, 256, "rows"), (12, 72, "heads"), (7, 24, "heads")])
def test_rows_to_pages_and_back(dtype, Hkv, d, order):
    c = U.make([1, 3, 0, 70, 5], [5, 40, 3, 71, 5], Hkv, Hkv, d, 16, dtype, order, seed=d)
    for seed in (0, 1):
        k, v = wild(c.T, Hkv * d, c.dtype, seed), wild(c.T, Hkv * d, c.dtype, seed + 2)
        got = G.append(c, k, v)
        assert got[2] == 0
        check_append(c, got, k, v)
        c.four = got[:2]
        ko, vo, st = G.read(c)
        assert st == 0
        for x, y in ((k, ko), (v, vo)):
            assert torch.equal(y.double().view(c.T, Hkv, d), U.unpack(U.pack(x.view(c.T, Hkv, d)), d))


def test_every_order_of_magnitude_and_what_is_no_number():
    c = U.make([520], [520], 1, 1, 32, 64, "f32", seed=1)
    g = torch.Generator().manual_seed(3)
    k = torch.randn((520, 32), generator=g).double()
    k /= k.abs().amax(-1, keepdim=True)
    k = (k * torch.exp2(torch.linspace(-149, 128, 520).double())[:, None]).clamp(-3.4028234e38, 3.4028234e38).float()
    v = k.clone()
    v[3, 5], v[7, 0], v[9, 31], v[11] = float("nan"), float("inf"), -float("inf"), 0.0
    v[12] = -0.0
    got = G.append(c, k, v)
    check_append(c, got, k, v)
    c.four = got[:2]
    ko, vo, _ = G.read(c)
    assert torch.isfinite(ko).all()
    for t in (3, 7, 9):
        assert torch.isnan(vo[t]).all()
    # the nearest of what the block's scale offers: half a unit of the largest binade at most, a unit where it is the largest
    unit = torch.exp2(U.pack(k)[1].double() - 127)
    assert bool(((ko.double() - k.double()).abs() <= torch.where(unit > 2.0 ** 124, 2.0, 1.0) * unit).all())


@pytest.mark.parametrize("many", [1500, 4000])
def test_many_tokens(many):
    c = U.make([many, 1, 200], [many + 7, 1, 300], 20, 20, 64, 64, "bf16", seed=2)
    k, v = wild(c.T, 20 * 64, c.dtype, 0), wild(c.T, 20 * 64, c.dtype, 2)
    got = G.append(c, k, v)
    check_append(c, got, k, v)
    c.four = got[:2]
    assert torch.equal(G.read(c)[0].double().view(c.T, 20, 64), U.unpack(U.pack(k.view(c.T, 20, 64)), 64))


def test_views_of_wider_rows_one_array_alone_and_tokens_without_a_key():
    c = U.make([2, 5, 1], [7, 5, 3], 4, 2, 64, 16, "bf16", seed=5)
    rows = wild(c.T, 3 * 128, c.dtype, 0).cuda()
    kp, vp = G.pool(c.four[0], "heads"), G.pool(c.four[1], "heads")
    st = G.status()
    kv = torch.tensor([7, 3, 3], dtype=torch.int32)  # (the second has more tokens than keys)
    cache = G.cache_of(c, kp, kv=kv)
    D.dart_append_4bit(cache, rows[:, :128], rows[:, 256:], kp, vp, status=st)
    assert int(st) == 1
    check_append(with_kv(c, [7, 3, 3]), (G.back(kp), G.back(vp)), rows[:, :128].cpu(),
                 rows[:, 256:].cpu())
    out = torch.full((c.T, 128), 7.0, dtype=c.dtype, device="cuda")
    D.dart_read_4bit(cache, None, vp, None, out)
    want = U.unpack(U.pack(rows[:, 256:].cpu().view(c.T, 2, 64)), 64).view(c.T, 128)
    want[2:7] = 7.0
    assert torch.equal(out.cpu().double(), want)
    D.dart_read_4bit(cache, None, None)  # nothing is asked for


def with_kv(c, kv):
    import copy
    d = copy.copy(c)
    d.kv = kv
    return d


def test_bad_pages_and_lengths_are_flagged_and_not_followed():
    c = U.make([2, 2], [20, 20], 2, 2, 64, 16, "bf16", seed=6)
    k, v = wild(4, 128, c.dtype, 0), wild(4, 128, c.dtype, 2)
    table = c.table.clone()
    table[0, 1] = 10 ** 6  # (the page of the first sequence's tokens)
    kp, vp, st = G.append(c, k, v, table=table)
    assert st == 2
    good = with_kv(c, [0, 20])
    check_append(good, (kp, vp), k, v)
    assert G.append(c, k, v, kv=torch.tensor([-1, 10 ** 6], dtype=torch.int32))[2] == 1
    assert G.attend(c, scale=0.1, table=table)[2] == 2


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 128), (7, 1, 128), (6, 2, 64), (2, 2, 80), (4, 1, 256), (3, 3, 8), (12, 4, 96), (20, 1, 40)])
@pytest.mark.parametrize("causal", [True, False])
def test_ragged_prompts(dtype, Hq, Hkv, d, causal):
    c = U.make(RAGGED_N, RAGGED_KV, Hq, Hkv, d, 16, dtype, seed=d, pad=8)
    out, lse, st = G.attend(c, scale=d ** -0.5, causal=causal, out_pad=16)
    assert st == 0
    A.check(c, (out, lse), scale=d ** -0.5, causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 128), (28, 4, 128), (8, 1, 64), (5, 5, 72), (16, 2, 256), (40, 1, 128)])
def test_one_token_of_each_sequence(dtype, Hq, Hkv, d):
    kv = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 700, 0, 1025]
    c = U.make([1] * len(kv), kv, Hq, Hkv, d, 16, dtype, seed=3)
    for packed in (False, True):
        A.check(c, G.attend(c, scale=0.1, packed=packed)[:2], scale=0.1)


@pytest.mark.parametrize("page", [1, 2, 16, 32, 256, 2048])
@pytest.mark.parametrize("order", ["heads", "rows"])
def test_pages_of_any_size_and_order(page, order):
    c = U.make([1, 40, 1, 7], [77, 40, 500, 1200], 6, 3, 64, page, "bf16", order, seed=page)
    A.check(c, G.attend(c, scale=0.125)[:2], scale=0.125)
    c = U.make([1, 1, 1], [333, 5, 1900], 6, 3, 64, page, "f32", order, seed=page)
    A.check(c, G.attend(c, scale=0.125)[:2], scale=0.125)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,kv", [([300], [300]), ([64], [3000]), ([1000], [90]), ([1, 1, 1], [9000, 1, 4097]), ([3, 1], [5000, 12001])])
def test_long_prompts_and_contexts(dtype, n, kv):
    c = U.make(n, kv, 8, 2, 128, 32, dtype, seed=n[0])
    A.check(c, G.attend(c, scale=0.09)[:2], scale=0.09)


@pytest.mark.parametrize("Hq,Hkv,d", [(32, 32, 128), (36, 36, 80), (40, 8, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_batches_that_fill_the_chip_with_rows(Hq, Hkv, d, causal):
    n = [1, 300, 257, 0, 64, 129, 512, 31, 255, 1, 400, 256, 200, 333, 65, 128, 300, 7, 450, 290, 256, 260, 37]
    kv = [9, 300, 300, 5, 0, 200, 512, 31, 100, 1, 400, 700, 200, 334, 65, 191, 301, 1500, 450, 290, 256, 292, 40]
    c = U.make(n, kv, Hq, Hkv, d, 64, "bf16", seed=Hq)
    A.check(c, G.attend(c, scale=d ** -0.5, causal=causal)[:2], scale=d ** -0.5, causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,n", [(4, 4, [1] * 9), (14, 2, [1] * 9), (4, 2, [5, 1, 0, 33, 2, 1, 70, 1, 8])])
@pytest.mark.parametrize("prefix", [[700, 0, 65], [1, 2500, 64]])
def test_shared_prefixes(dtype, Hq, Hkv, n, prefix):
    kv = [a + b for a, b in zip(n, [0, 3, 64, 100, 17, 0, 31, 250, 9])]
    c = U.make(n, kv, Hq, Hkv, 128, 16, dtype, groups=[4, 2, 3], prefix=prefix, seed=7)
    A.check(c, G.attend(c, scale=0.0884)[:2], scale=0.0884)


def test_scales_of_either_sign_and_rows_that_see_nothing():
    c = U.make([1, 20, 6], [90, 150, 2], 4, 2, 64, 16, "bf16", seed=6)
    for scale in (-0.3, 0.0, 1.0):
        A.check(c, G.attend(c, scale=scale)[:2], scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_that_are_no_number_show_where_they_are_seen(dtype):
    c = U.make([70, 1], [130, 40], 4, 2, 96, 16, dtype, seed=9)
    want, want_lse, tol, lse_tol = A.reference(c, 0.1, True)
    page, row = U.places(c, 0)
    c.four[1][1][page[100], 1, row[100], 1] = 255  # values 32..63 of key 100, head 1: seen by tokens 40 on
    c.four[0][1][page[120], 0, row[120], 0] = 255  # a key of head 0: seen by tokens 60 on
    out, lse, _ = G.attend(c, scale=0.1)
    bad = torch.zeros(out.shape, dtype=torch.bool)
    bad[40:70, 2:, 32:64] = True
    bad[60:70, :2] = True
    assert torch.isnan(out[bad].float()).all()
    assert bool(((out.double() - want).abs() <= tol)[~bad].all())
    odd = torch.zeros(lse.shape, dtype=torch.bool)
    odd[60:70, :2] = True
    assert torch.isnan(lse[odd]).all() and bool(((lse.double() - want_lse).abs() <= lse_tol)[~odd].all())


def test_the_same_values_as_rows_give_the_same_results():
    """bf16 rows hold every 4-bit value, so attention over either pool has the same products."""
    c = U.make([40, 1, 9], [200, 700, 9], 8, 2, 128, 16, "bf16", seed=4)
    out, lse, _ = G.attend(c, scale=0.09)
    rows, rows_lse = A.attend(c, scale=0.09)
    want, want_lse, tol, lse_tol = A.reference(c, 0.09, True)
    assert bool(((out.double() - rows.double()).abs() <= 2 * tol).all()) and bool(((lse - rows_lse).abs() <= 2 * lse_tol).all())


def test_without_lse_and_on_another_stream():
    c = U.make([3, 1], [100, 900], 8, 2, 128, 16, "bf16", seed=11)
    kp, vp = G.pool(c.four[0], c.order), G.pool(c.four[1], c.order)
    cache = G.cache_of(c, kp)
    ws, q = D.alloc_attend_4bit_workspace(cache), A.to_gpu(c.q)
    out = torch.empty((c.T, 8 * 128), dtype=c.dtype, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    D.dart_attend_4bit(cache, q, kp, vp, out, ws, scale=0.09, stream=side)
    side.synchronize()
    A.check(c, (out.cpu().view(c.T, 8, 128), None), scale=0.09)


def test_a_graph_of_append_and_attention_follows_the_tensors_it_names():
    c = U.make([1, 1, 1], [100, 17, 900], 8, 2, 128, 16, "bf16", seed=12)
    kp, vp = G.pool(c.four[0], c.order), G.pool(c.four[1], c.order)
    cache = G.cache_of(c, kp)
    ws, q = D.alloc_attend_4bit_workspace(cache), A.to_gpu(c.q)
    k, v = (wild(3, 256, c.dtype, s).cuda() for s in (0, 2))
    out = torch.empty((3, 1024), dtype=c.dtype, device="cuda")

    def step():
        D.dart_append_4bit(cache, k, v, kp, vp)
        D.dart_attend_4bit(cache, q, kp, vp, out, ws, scale=0.09)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (4, 6, 8):
        k.copy_(wild(3, 256, c.dtype, seed))
        v.copy_(wild(3, 256, c.dtype, seed + 10))
        q.copy_(torch.randn((3, 1024), generator=torch.Generator().manual_seed(seed)).to(c.dtype))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out)
