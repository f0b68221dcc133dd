"""Attention over the paged cache against its definition in 64 bits, at the sizes, masks, orders and
contents where it can go wrong.  The tolerance of every element is derived from the stated arithmetic
(attend_util.reference)."""
import pytest
import torch

import paper_2502_11494_amd as D

import attend_util as A

pytestmark = pytest.mark.gpu


# sequences with no token, no key, fewer keys than tokens (rows that see nothing), one key, and lengths
# on both sides of every tile and page boundary
RAGGED_N = [1, 0, 3, 17, 1, 64, 33, 5, 1, 130]
RAGGED_KV = [1, 9, 3, 40, 0, 65, 20, 128, 300, 257]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 128), (7, 1, 128), (6, 2, 64), (2, 2, 80), (4, 1, 256), (3, 3, 8), (12, 4, 96),
                                      (20, 1, 40)])
@pytest.mark.parametrize("causal", [True, False])
def test_ragged_prompts(dtype, Hq, Hkv, d, causal):
    c = A.make(RAGGED_N, RAGGED_KV, Hq, Hkv, d, 16, dtype, seed=d, pad=8)
    A.check(c, A.attend(c, scale=d ** -0.5, causal=causal, out_pad=16), scale=d ** -0.5, causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 128), (28, 4, 128), (8, 1, 64), (5, 5, 72), (16, 2, 256), (40, 1, 128)])
def test_one_token_of_each_sequence(dtype, Hq, Hkv, d):
    kv = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 700, 0, 1025]
    c = A.make([1] * len(kv), kv, Hq, Hkv, d, 16, dtype, seed=3)
    for packed in (False, True):
        A.check(c, A.attend(c, scale=0.1, packed=packed), scale=0.1)


@pytest.mark.parametrize("page", [1, 2, 16, 32, 256, 2048])
@pytest.mark.parametrize("order", ["heads", "rows"])
def test_pages_of_any_size_and_order(page, order):
    c = A.make([1, 40, 1, 7], [77, 40, 500, 1200], 6, 3, 64, page, "bf16", order, seed=page)
    A.check(c, A.attend(c, scale=0.125), scale=0.125)
    c = A.make([1, 1, 1], [333, 5, 1900], 6, 3, 64, page, "f32", order, seed=page)
    A.check(c, A.attend(c, scale=0.125), scale=0.125)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,kv", [(300, 300), (257, 1000), (64, 3000), (600, 600), (1000, 90)])
def test_long_prompts(dtype, n, kv):
    c = A.make([n], [kv], 4, 2, 128, 64, dtype, seed=n)
    A.check(c, A.attend(c, scale=0.09), scale=0.09)


@pytest.mark.parametrize("Hq,Hkv,d", [(32, 32, 128), (32, 32, 64), (36, 36, 80), (40, 8, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_batches_that_fill_the_chip_with_rows(Hq, Hkv, d, causal):
    """Batches of rows enough for the widest tiles (more than 256 of a key head for every unit twice): sequences that end
    inside a tile, start inside one, see one key, fewer keys than they have tokens, or none."""
    n = [1, 300, 257, 0, 64, 129, 512, 31, 255, 1, 400, 256, 200, 333, 65, 128, 300, 7, 450, 290, 256, 260, 37]
    kv = [9, 300, 300, 5, 0, 200, 512, 31, 100, 1, 400, 700, 200, 334, 65, 191, 301, 500, 450, 290, 256, 292, 40]
    assert sum(n) * (Hq // Hkv) // 256 * Hkv >= 512 and max(n) * (Hq // Hkv) > 128
    c = A.make(n, kv, Hq, Hkv, d, 64, "bf16", seed=Hq)
    A.check(c, A.attend(c, scale=d ** -0.5, causal=causal), scale=d ** -0.5, causal=causal)


def test_odd_values_in_batches_that_fill_the_chip_with_rows():
    n = [300, 257, 64, 129, 512, 31, 255, 400, 256, 200, 333, 65, 128, 300, 450, 290, 256, 260]
    c = A.make(n, n, 32, 32, 64, 64, "bf16", seed=3)
    want, want_lse, tol, lse_tol = A.reference(c, 0.125, True)
    for b, at, value in ((1, 70, float("nan")), (4, 300, float("inf")), (4, 333, -float("inf")), (9, 0, float("nan"))):
        c.v_pool[int(c.table[b, at // 64]), 5, at % 64] = value
    out, lse = A.attend(c, scale=0.125)
    ok = torch.ones((c.T, 32), dtype=torch.bool)
    for b, at in ((1, 70), (4, 300), (9, 0)):
        ok[int(c.cu[b]) + at:int(c.cu[b + 1]), 5] = False
    assert bool(((out.double() - want).abs() <= tol)[ok].all())
    assert bool(((lse.double() - want_lse).abs() <= lse_tol).all())
    o = out.float()[:, 5]
    first = [int(x) for x in c.cu]
    assert torch.isnan(o[first[1] + 70:first[2]]).all() and torch.isnan(o[first[9]:first[10]]).all()
    assert bool((o[first[4] + 300:first[4] + 333] == float("inf")).all()) and torch.isnan(o[first[4] + 333:first[5]]).all()


@pytest.mark.parametrize("n,kv", [([1, 1, 1], [9000, 1, 4097]), ([3, 1], [5000, 12001]), ([1], [20011])])
def test_long_contexts_of_few_rows(n, kv):
    """The work of a few rows is split along the keys and joined."""
    for dtype in ("bf16", "f32"):
        c = A.make(n, kv, 8, 2, 128, 32, dtype, seed=1)
        A.check(c, A.attend(c, scale=0.09), scale=0.09)


@pytest.mark.parametrize("spread", [1e-3, 12.0])
def test_flat_and_peaked_scores(spread):
    for dtype in ("bf16", "f32"):
        c = A.make([1, 50, 1], [700, 50, 2100], 4, 2, 128, 16, dtype, seed=5, spread=spread)
        A.check(c, A.attend(c, scale=0.0884), scale=0.0884)


def test_scale_of_either_sign_and_zero():
    c = A.make([1, 20], [90, 150], 4, 2, 64, 16, "bf16", seed=6)
    for scale in (-0.3, 0.0, 1.0):
        A.check(c, A.attend(c, scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,n", [(4, 4, [1] * 9), (14, 2, [1] * 9), (4, 2, [5, 1, 0, 33, 2, 1, 70, 1, 8])])
@pytest.mark.parametrize("prefix", [[700, 0, 65], [1, 2500, 64]])
def test_shared_prefixes(dtype, Hq, Hkv, n, prefix):
    kv = [a + b for a, b in zip(n, [0, 3, 64, 100, 17, 0, 31, 250, 9])]
    c = A.make(n, kv, Hq, Hkv, 128, 16, dtype, groups=[4, 2, 3], prefix=prefix, seed=7)
    A.check(c, A.attend(c, scale=0.0884), scale=0.0884)


@pytest.mark.parametrize("causal", [True, False])
def test_prefix_of_a_group_without_sequences_and_sequences_without_keys(causal):
    n, kv = [1, 3, 2, 1, 4], [0, 1, 0, 5, 4]  # (rows that see the prefix and nothing of their own)
    c = A.make(n, kv, 6, 2, 64, 32, "bf16", groups=[2, 0, 3], prefix=[40, 999, 0], seed=8)
    A.check(c, A.attend(c, scale=0.2, causal=causal), scale=0.2, causal=causal)


def test_prefix_equals_the_same_keys_in_front():
    """A shared prefix gives what a cache with the prefix in front of every sequence gives."""
    c = A.make([1] * 6, [20, 1, 64, 33, 90, 7], 8, 2, 128, 16, "f32", groups=[6], prefix=[333], seed=9)
    out, lse = A.attend(c, scale=0.1)
    whole = A.make([1] * 6, [x + 333 for x in c.kv], 8, 2, 128, 16, "f32", seed=9)
    whole.q = c.q
    for b, x in enumerate(c.kv):
        for pool, src in ((whole.k_pool, c.k_pool), (whole.v_pool, c.v_pool)):
            for h in range(2):
                rows = torch.cat((A.keys_of(c, src, c.front[0], 333, h), A.keys_of(c, src, c.table[b], x, h))).float()
                w = torch.arange(x + 333)
                pool[whole.table[b].long()[w // 16], h, w % 16] = rows
    A.check(whole, (out, lse), scale=0.1)


def test_what_lies_after_a_token_is_not_used_even_when_it_is_no_number():
    """Infinities and NaN in the keys and values of later tokens reach those tokens and no earlier one."""
    for dtype in ("bf16", "f32"):
        for d in (64, 128):
            for at, kv in ((70, 100), (31, 40), (64, 200), (0, 3)):
                c = A.make([kv], [kv], 4, 2, d, 16, dtype, seed=at)
                clean = A.reference(c, 0.1, True)
                p, r = int(c.table[0, at // 16]), at % 16
                for what, value in (("k", float("nan")), ("v", float("nan")), ("v", float("inf")), ("v", -float("inf"))):
                    pool = c.k_pool if what == "k" else c.v_pool
                    keep = pool[p, 1, r].clone()
                    pool[p, 1, r] = value
                    out, lse = A.attend(c, scale=0.1)
                    pool[p, 1, r] = keep
                    ok = torch.ones((c.T, c.Hq), dtype=torch.bool)
                    ok[at:, 2:] = False  # the tokens from there on, in the heads that read key head 1
                    err = (out.double() - clean[0]).abs()
                    assert bool((err[ok] <= clean[2][ok]).all()), (dtype, d, at, what, value)
                    hit = out[at:, 2:].float()
                    if what == "k" or value != value:
                        assert torch.isnan(hit).all()
                    else:
                        assert bool((hit == value).all())
                    if what == "v":
                        assert bool(((lse.double() - clean[1]).abs() <= clean[3]).all())


def test_scores_of_minus_infinity_weigh_nothing():
    c = A.make([1, 1], [40, 3], 2, 1, 64, 16, "bf16", seed=2)
    c.q[:] = c.q.abs()
    for b, rows in ((0, [0, 7, 39]), (1, [0, 1, 2])):
        for j in rows:
            c.k_pool[int(c.table[b, j // 16]), 0, j % 16] = -float("inf")
    out, lse = A.attend(c, scale=0.1)
    assert bool((out[1] == 0).all()) and bool((lse[1] == -float("inf")).all())
    for j in (39, 7, 0):  # the same without those keys
        for i in range(j, 39):
            for pool in (c.k_pool, c.v_pool):
                pool[int(c.table[0, i // 16]), 0, i % 16] = pool[int(c.table[0, (i + 1) // 16]), 0, (i + 1) % 16]
    c.kv = [37, 0]
    want, want_lse, tol, lse_tol = A.reference(c, 0.1, True)
    assert bool(((out.double() - want).abs() <= tol)[0].all())
    assert bool(((lse.double() - want_lse).abs() <= lse_tol)[0].all())


def test_offsets_past_32_bits():
    """Pages 2^30 elements apart: the last lies 6 GB into its pool."""
    for dtype, apart in (("bf16", 1 << 30), ("f32", 1 << 29)):
        c = A.make([1, 9], [50, 70], 4, 2, 64, 16, dtype, seed=4)
        pages = c.k_pool.shape[0]
        pools = []
        for src in (c.k_pool, c.v_pool):
            room = torch.empty(apart * (pages - 1) + src[0].numel(), dtype=src.dtype, device="cuda")
            pool = room.as_strided(src.shape, (apart, 16 * 64, 64, 1))
            pool.copy_(src.cuda())
            pools.append(pool)
        assert apart * (pages - 1) > 2 ** 32
        A.check(c, A.attend(c, scale=0.1, k_pool=pools[0], v_pool=pools[1]), scale=0.1)


def test_bad_sequences_are_skipped_and_flagged():
    kv = [50, 60, 70, 80]
    c = A.make([2, 3, 4, 5], kv, 4, 2, 64, 16, "bf16", seed=10)
    want = A.attend(c, scale=0.1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    A.attend(c, scale=0.1, status=status)
    assert int(status) == 0

    def skipped(b, bit, **how):
        status.zero_()
        out, lse = A.attend(c, scale=0.1, status=status, **how)
        assert int(status) & bit
        rows = slice(int(c.cu[b]), int(c.cu[b + 1]))
        others = torch.ones(c.T, dtype=torch.bool)
        others[rows] = False
        assert torch.equal(out[others], want[0][others]) and torch.equal(lse[others], want[1][others])
        return out[rows], lse[rows]

    long = torch.tensor([50, 60, 7000, 80], dtype=torch.int32)
    for kv_len in (long, torch.tensor([50, 60, -1, 80], dtype=torch.int32)):
        out, lse = skipped(2, 1, kv=kv_len)
        assert bool((out == 0).all()) and bool((lse == -float("inf")).all())
    out, lse = skipped(2, 1, kv=long, max_kv=8000)  # (more keys than the table has room for)
    assert bool((out == 0).all())
    out, lse = skipped(3, 1, max_q=4)
    assert bool((out == 0).all())
    table = c.table.clone()
    for page in (-1, c.k_pool.shape[0], 2 ** 31 - 1):
        table[1, 2] = page
        skipped(1, 2, table=table)


def test_bad_prefixes_and_offsets_are_flagged():
    c = A.make([1, 2, 3], [9, 9, 9], 4, 2, 64, 16, "bf16", groups=[1, 2], prefix=[30, 40], seed=11)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = A.attend(c, scale=0.1)
    c.prefix = [30, 4000]
    bad = A.cache_of(c, A.pool_to_gpu(c.k_pool, "heads"))
    assert bad.max_prefix == 4000
    out, lse = A.attend(c, scale=0.1, status=status)  # (more than the table has room for)
    assert int(status) == 1 and bool((out[1:] == 0).all()) and torch.equal(out[:1], want[0][:1])
    c.prefix = [30, 40]
    for cu in ([0, 1, 0, 6], [0, 1, 9, 6], [-5, 1, 3, 6], [3, 1, 3, 6]):  # nothing is read or written out of bounds
        status.zero_()
        A.attend(c, scale=0.1, status=status, cu=torch.tensor(cu, dtype=torch.int32))
        assert int(status) == 1


def test_calls_without_tokens():
    c = A.make([1], [5], 4, 2, 64, 16, "bf16")
    pool = c.k_pool.cuda()
    none = D.make_cache(4, pool, torch.zeros((0, 1), dtype=torch.int32, device="cuda"),
                        torch.zeros(0, dtype=torch.int32, device="cuda"), 0)
    empty = torch.empty((0, 256), dtype=torch.bfloat16, device="cuda")
    D.dart_attend(none, empty, pool, pool, empty, D.alloc_attend_workspace(none), scale=1.0)
    c = A.make([0, 0], [5, 0], 4, 2, 64, 16, "bf16")
    cache = D.make_cache(4, pool, c.table.cuda(), torch.tensor([5, 0], dtype=torch.int32).cuda(), 5, T=0, max_q=0,
                         cu_q=c.cu.cuda())
    D.dart_attend(cache, empty, pool, pool, empty, D.alloc_attend_workspace(cache), scale=1.0)
    torch.cuda.synchronize()


def test_same_inputs_same_bits_on_any_stream_and_in_a_graph():
    c = A.make([1, 40, 1, 9], [4000, 300, 77, 900], 8, 2, 128, 16, "bf16", groups=[3, 1], prefix=[500, 20], seed=12)
    first = A.attend(c, scale=0.1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = A.attend(c, scale=0.1, ws_fill=0, stream=side)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    k_pool, v_pool = c.k_pool.cuda(), c.v_pool.cuda()
    cache = A.cache_of(c, k_pool)
    ws, q = D.alloc_attend_workspace(cache), A.to_gpu(c.q)
    out, lse = torch.empty((c.T, 1024), dtype=torch.bfloat16, device="cuda"), torch.empty((c.T, 8), device="cuda")
    call = lambda: D.dart_attend(cache, q, k_pool, v_pool, out, ws, scale=0.1, lse=lse)  # noqa: E731
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        out.fill_(3)
        lse.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu().view(c.T, 8, 128), first[0]) and torch.equal(lse.cpu(), first[1])


def test_more_sequences_and_groups_than_lanes_of_a_wave():
    """The join then looks its rows' sequences and groups up by searches."""
    n = [i % 3 for i in range(72)]
    kv = [a + i * 53 % 600 for i, a in enumerate(n)]
    c = A.make(n, kv, 4, 1, 64, 16, "bf16", seed=72)
    A.check(c, A.attend(c, scale=0.125), scale=0.125)
    groups = [1] * 60 + [2] * 6
    c = A.make(n, kv, 4, 2, 64, 16, "bf16", groups=groups, prefix=[i * 37 % 300 for i in range(66)], seed=73)
    A.check(c, A.attend(c, scale=0.125), scale=0.125)
    c = A.make([1] * 72, [1 + x for x in kv], 4, 1, 64, 16, "f32", groups=groups, prefix=[i * 37 % 300 for i in range(66)], seed=74)
    A.check(c, A.attend(c, scale=0.125), scale=0.125)


@pytest.mark.parametrize("Hq,Hkv,d", [(32, 32, 128), (32, 32, 64), (36, 36, 80), (40, 8, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_batches_that_fill_the_chip_with_rows_and_may_have_long_contexts(Hq, Hkv, d, causal):
    """The bound on the keys, not the keys, chooses the widest tiles: sequences as above and one of 1100 keys."""
    n = [1, 300, 257, 0, 64, 129, 512, 31, 255, 1, 400, 256, 200, 333, 65, 128, 300, 7, 450, 290, 256, 260, 37]
    kv = [9, 300, 300, 5, 0, 200, 512, 31, 100, 1, 400, 700, 200, 334, 65, 191, 301, 1100, 450, 290, 256, 292, 40]
    c = A.make(n, kv, Hq, Hkv, d, 64, "bf16", seed=Hq + 1)
    A.check(c, A.attend(c, scale=d ** -0.5, causal=causal, max_kv=5000), scale=d ** -0.5, causal=causal)


def test_odd_values_in_the_widest_tiles():
    n = [300, 257, 64, 129, 512, 31, 255, 400, 256, 200, 333, 65, 128, 300, 450, 290, 256, 260]
    c = A.make(n, n, 32, 32, 64, 64, "bf16", seed=4)
    want, want_lse, tol, lse_tol = A.reference(c, 0.125, True)
    for b, at, value in ((1, 70, float("nan")), (4, 300, float("inf"))):
        c.v_pool[int(c.table[b, at // 64]), 5, at % 64] = value
    out, lse = A.attend(c, scale=0.125, max_kv=5000)
    ok = torch.ones((c.T, 32), dtype=torch.bool)
    for b, at in ((1, 70), (4, 300)):
        ok[int(c.cu[b]) + at:int(c.cu[b + 1]), 5] = False
    assert bool(((out.double() - want).abs() <= tol)[ok].all())
    assert bool(((lse.double() - want_lse).abs() <= lse_tol).all())
    o, first = out.float()[:, 5], [int(x) for x in c.cu]
    assert torch.isnan(o[first[1] + 70:first[2]]).all()
    assert bool((o[first[4] + 300:first[5]] == float("inf")).all())


@pytest.mark.parametrize("dtype,n,Hq,Hkv,prefix,groups", [
    ("bf16", [500, 1, 700, 450, 0, 600, 513, 800], 28, 28, [1100, 64], [3, 5]),   # the widest tiles over the prefixes
    ("f32", [40, 33, 1, 70] * 8, 16, 16, [300, 0, 511, 64], [9, 7, 8, 8]),          # prefixes and own keys in two launches
])
def test_prefixes_of_many_rows(dtype, n, Hq, Hkv, prefix, groups):
    kv = [x + i % 5 * 13 for i, x in enumerate(n)]
    c = A.make(n, kv, Hq, Hkv, 64, 32, dtype, groups=groups, prefix=prefix, seed=len(n))
    for causal in (True, False):
        A.check(c, A.attend(c, scale=0.125, causal=causal), scale=0.125, causal=causal)
