"""Gathered attention weights against their definition in 64 bits, with tolerances derived from the stated arithmetic
(more_util.gathered), and eviction bit for bit against a sort."""
import pytest
import torch

import attend_util as A
import more_gpu as G
import more_util as U
import paper_2502_11494_amd as D

pytestmark = pytest.mark.gpu

RAGGED_N = [1, 0, 3, 17, 1, 64, 33, 5, 1, 130]
RAGGED_KV = [1, 9, 3, 40, 0, 65, 20, 128, 300, 257]


def old_weights(c, seed=1):
    pages, Hkv = c.k_pool.shape[:2]
    return torch.rand((pages, Hkv, c.page), generator=torch.Generator().manual_seed(seed))


def run(c, scale, causal=True, carry=1.0, **how):
    lse = A.reference(c, scale, causal)[1].float()
    old = old_weights(c)
    got, st = G.weights(c, lse, old, scale=scale, causal=causal, carry=carry, **how)
    assert st == 0
    U.check_gathered(c, got, lse, old, scale=scale, causal=causal, carry=carry)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 128), (7, 1, 128), (6, 2, 64), (2, 2, 80), (4, 1, 256), (3, 3, 8), (12, 4, 96), (20, 1, 40)])
@pytest.mark.parametrize("causal", [True, False])
def test_weights_of_ragged_prompts(four, dtype, Hq, Hkv, d, causal):
    run(U.make(RAGGED_N, RAGGED_KV, Hq, Hkv, d, 16, dtype, seed=d, pad=8, four=four), d ** -0.5, causal, 0.5)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d", [(28, 4, 128), (8, 1, 64), (5, 5, 72), (16, 2, 256)])
def test_weights_of_one_token_each(four, dtype, Hq, Hkv, d):
    kv = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 700, 0, 1025]
    c = U.make([1] * len(kv), kv, Hq, Hkv, d, 16, dtype, seed=3, four=four)
    for packed in (False, True):
        run(c, 0.1, packed=packed)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("order", ["heads", "rows"])
@pytest.mark.parametrize("page", [1, 16, 2048])
def test_weights_in_pages_of_any_size_and_order(four, order, page):
    run(U.make([1, 40, 1, 7], [77, 40, 500, 1200], 6, 3, 64, page, "bf16", order, seed=page, four=four), 0.125, max_kv=5000)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,kv", [([1200], [1200]), ([700], [2000]), ([1000], [90]), ([900, 5], [950, 3000])])
def test_weights_of_long_prompts(dtype, n, kv):
    """The rows are dealt to several blocks, whose sums are joined."""
    c = U.make(n, kv, 4, 1, 128, 64, dtype, seed=n[0], four=False)
    for causal, carry in ((True, 0.0), (False, 1.0)):
        run(c, 0.09, causal, carry)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [[1] * 9, [5, 1, 0, 33, 2, 1, 70, 1, 8], [200, 100, 0, 1, 1, 0, 0, 3, 260]])
def test_weights_of_shared_prefixes(four, dtype, n):
    kv = [a + b for a, b in zip(n, [0, 3, 64, 100, 17, 0, 31, 250, 9])]
    run(U.make(n, kv, 14, 2, 64, 16, dtype, groups=[4, 0, 2, 3], prefix=[700, 9, 65, 300], seed=7, four=four), 0.125, carry=0.9)


def test_weights_with_scales_of_either_sign_and_rows_that_see_nothing():
    c = U.make([1, 20, 6], [90, 150, 2], 4, 2, 64, 16, "bf16", seed=6, four=False)
    for scale in (-0.3, 0.0, 1.0):
        run(c, scale)


def test_weights_are_not_read_where_they_do_not_count():
    c = U.make([3, 1], [40, 300], 4, 2, 64, 16, "bf16", seed=2, four=False)
    lse = A.reference(c, 0.1, True)[1].float()
    want = G.weights(c, lse, old_weights(c), scale=0.1, carry=0.0)[0]
    nan = torch.full_like(want, float("nan"))
    got = G.weights(c, lse, nan, scale=0.1, carry=0.0)[0]
    for b in range(2):
        page, row = U.places(c, b)
        assert torch.equal(got[page, :, row], want[page, :, row])
    # (and those of the call's own keys are not, whatever carry is)
    old = old_weights(c)
    page, row = U.places(c, 0)
    old[page[-3:], :, row[-3:]] = float("nan")
    assert torch.isfinite(G.weights(c, lse, old, scale=0.1, carry=0.7)[0][page, :, row]).all()


def test_a_key_that_is_no_number_spoils_its_own_weight_only():
    c = U.make([40], [100], 2, 2, 64, 16, "bf16", seed=4, four=False)
    lse = A.reference(c, 0.1, True)[1].float()
    old = old_weights(c)
    page, row = U.places(c, 0)
    c.k_pool[page[70], 1, row[70], 3] = float("nan")
    c.k_pool[page[99], 0, row[99], 3] = float("inf")
    got = G.weights(c, lse, old, scale=0.1)[0]
    assert torch.isnan(got[page[70], 1, row[70]])
    got[page[70], 1, row[70]] = got[page[99], 0, row[99]] = 0
    assert torch.isfinite(got).all()


def test_wrong_sequences_and_pages_are_flagged_and_left():
    c = U.make([2, 2, 2], [20, 20, 20], 2, 2, 64, 16, "bf16", groups=[2, 1], prefix=[40, 30], seed=6, four=False)
    lse, old = A.reference(c, 0.1, True)[1].float(), old_weights(c)
    good = G.weights(c, lse, old, scale=0.1)[0]
    kv = torch.tensor([20, -4, 20], dtype=torch.int32)
    kp = A.pool_to_gpu(c.k_pool, c.order)
    cache = A.cache_of(c, kp, kv=kv)
    w, st = old.cuda(), G.status()
    D.dart_attend_weights(cache, A.to_gpu(c.q), kp, lse.cuda(), w, D.alloc_attend_weights_workspace(cache), scale=0.1, status=st)
    w = w.cpu()
    assert int(st) == 1
    for b, same in ((0, good), (1, old), (2, good)):
        page, row = U.places(c, b)
        assert torch.equal(w[page, :, row], same[page, :, row])
    for g, same in ((0, old), (1, good)):  # (the group of the skipped sequence is skipped)
        page, row = U.places(c, None, c.prefix[g], c.front[g])
        assert torch.equal(w[page, :, row], same[page, :, row])
    table = c.table.clone()
    table[2, 0] = -7
    assert G.weights(c, lse, old, scale=0.1, table=table)[1] == 2


# ---- eviction ---------------------------------------------------------------------------------

KV = [0, 1, 2, 30, 31, 64, 100, 333, 1024, 1500]


def worth(c, seed, kind="spread"):
    g = torch.Generator().manual_seed(seed)
    pages, Hkv = c.k_pool.shape[:2]
    w = torch.randn((pages, Hkv, c.page), generator=g)
    if kind == "ties":
        w = (w * 2).round()
    elif kind == "alike":
        w = torch.ones_like(w)
    elif kind == "odd":
        odd = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45, -1e-45, 3.4e38])
        w = odd[torch.randint(0, 8, w.shape, generator=g)]
    elif kind == "spread":
        w = torch.exp(6 * w)
    return w


@pytest.mark.parametrize("kind", ["spread", "ties", "alike", "odd"])
@pytest.mark.parametrize("how", [dict(budget=30), dict(ratio=(111, 1000), first=3, recent=5), dict(ratio=(1, 2)), dict(budget=1),
                                 dict(ratio=(0, 1), first=2), dict(ratio=(1, 1)), dict(ratio=(0, 1)), dict(budget=7, first=60, recent=40)])
def test_kept_keys_and_their_rows(kind, how):
    c = U.make([0] * len(KV), KV, 2, 2, 64, 16, "bf16", seed=1, four=False)
    w = worth(c, 2, kind)
    got = G.evict(c, w, **how)
    assert got[4] == 0
    U.check_evicted(c, got[:4], w, **how)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv,d,page,order", [(4, 128, 16, "heads"), (1, 8, 1, "heads"), (3, 40, 64, "rows"), (2, 80, 2048, "heads"),
                                              (2, 256, 32, "rows"), (12, 96, 16, "heads"), (2, 72, 2, "rows")])
def test_rows_of_every_kind_move(four, dtype, Hkv, d, page, order):
    c = U.make([0] * 4, [500, 1, 130, 2100], Hkv, Hkv, d, page, dtype, order, seed=d, four=four)
    w = worth(c, d)
    for how in (dict(budget=129, first=1, recent=2), dict(ratio=(7, 10))):
        for out, keep, alias in (("other", True, False), ("same", False, True), (None, True, False)):
            got = G.evict(c, w, out=out, keep=keep, alias_len=alias, **how)
            assert got[4] == 0
            U.check_evicted(c, got[:4], w, **how)


@pytest.mark.parametrize("n", [16383, 16384, 16385, 16390 + 16384, 40000])
@pytest.mark.parametrize("kind", ["spread", "ties", "alike"])
def test_long_sequences(n, kind):
    c = U.make([0, 0], [n, 700], 1, 1, 8, 256, "bf16", seed=1, four=False)
    w = worth(c, n, kind)
    for how in (dict(budget=1500), dict(ratio=(9, 10), first=4, recent=100)):
        U.check_evicted(c, G.evict(c, w, **how)[:4], w, **how)


def test_many_sequences():
    kv = [1 + 7 * i % 90 for i in range(700)]
    c = U.make([0] * 700, kv, 3, 3, 16, 8, "bf16", seed=1, four=True)
    w = worth(c, 5)
    U.check_evicted(c, G.evict(c, w, budget=20, recent=3)[:4], w, budget=20, recent=3)


def test_bounds_over_the_lengths_and_wrong_lengths_and_pages():
    c = U.make([0] * 3, [100, 200, 300], 2, 2, 64, 16, "bf16", seed=1, four=False)
    w = worth(c, 1)
    U.check_evicted(c, G.evict(c, w, budget=50, max_kv=304)[:4], w, budget=50)
    pools, _, kept, left, st = G.evict(c, w, budget=50, kv=torch.tensor([100, -3, 301], dtype=torch.int32), max_kv=300)
    assert st == 1 and left.tolist() == [50, -3, 301]
    for b in (1, 2):
        page, row = U.places(c, b)
        for x, y in zip(pools, (c.k_pool, c.v_pool)):
            assert torch.equal(x[page, :, row].float(), y[page, :, row].float())
    table = c.table.clone()
    table[1, 3] = 1 << 20
    pools, _, kept, left, st = G.evict(c, w, budget=50, table=table)
    assert st == 2 and left.tolist() == [50, 50, 50]
    for b in (0, 2):  # (the others are cut as always)
        page, row = U.places(c, b)
        for h in range(2):
            src = kept[b, h].long()
            assert torch.equal(pools[0][page[:50], h, row[:50]], c.k_pool[page[src], h, row[src]])
    assert not bool(((kept[1] >= 48) & (kept[1] < 64)).any())


def test_the_calls_together_as_an_answer_uses_them():
    """A prompt into 4-bit pages, its weights, eviction, then answer tokens over what is left, against the same in 64 bits."""
    torch.manual_seed(0)
    Hq, Hkv, d, page, n, scale = 8, 2, 64, 16, [90, 40, 133], 0.125
    lens, room = list(n), 12
    table = torch.arange(3 * room, dtype=torch.int32).view(3, room)
    pools = [D.alloc_pool_4bit(3 * room, Hkv, page, d) for _ in range(2)]
    weights = torch.zeros((3 * room, Hkv, page), device="cuda")
    model = [[([], []) for _ in range(Hkv)] for _ in n]   # keys and values of each head, as the pages hold them
    gathered = [[torch.zeros(0, dtype=torch.float64) for _ in range(Hkv)] for _ in n]
    kv_len, st = torch.zeros(3, dtype=torch.int32, device="cuda"), G.status()
    eviction = D.make_eviction(budget=32, first=2, recent=8)
    for step in range(5):
        m = n if step == 0 else [1, 1, 1]
        T = sum(m)
        q, k, v = ((torch.randn((T, h * d)) * 1.3).bfloat16() for h in (Hq, Hkv, Hkv))
        kv_len += torch.tensor(m, dtype=torch.int32, device="cuda")
        cu = torch.tensor([sum(m[:i]) for i in range(4)], dtype=torch.int32)
        cache = D.make_cache_4bit(Hq, d, D.DART_BF16, pools[0], table.cuda(), kv_len, 160, T=T, max_q=max(m), cu_q=cu.cuda())
        out, lse = torch.empty((T, Hq * d), dtype=torch.bfloat16, device="cuda"), torch.empty((T, Hq), device="cuda")
        qg = q.cuda()
        D.dart_append_4bit(cache, k.cuda(), v.cuda(), *pools, status=st)
        D.dart_attend_4bit(cache, qg, *pools, out, D.alloc_attend_4bit_workspace(cache), scale=scale, lse=lse, status=st)
        D.dart_attend_weights(cache, qg, pools[0], lse, weights, D.alloc_attend_weights_workspace(cache), scale=scale, carry=0.9, status=st)
        ws = D.alloc_evict_workspace(cache, eviction)
        kept = torch.full((3, Hkv, D.dart_evict_most(cache, eviction)), -1, dtype=torch.int32, device="cuda")
        before = weights.clone().cpu()
        D.dart_evict(cache, eviction, *pools, weights, kv_len, ws, weights_out=weights, kept=kept, status=st)
        torch.cuda.synchronize()
        assert int(st) == 0
        for b in range(3):
            t = slice(int(cu[b]), int(cu[b + 1]))
            for h in range(Hkv):
                keys, values = model[b][h]
                keys += list(U.unpack(U.pack(k[t].view(-1, Hkv, d)[:, h]), d))
                values += list(U.unpack(U.pack(v[t].view(-1, Hkv, d)[:, h]), d))
                K, V = torch.stack(keys), torch.stack(values)
                total = torch.cat((0.9 * gathered[b][h], torch.zeros(m[b], dtype=torch.float64)))
                for x in range(h * 4, h * 4 + 4):
                    s = q[t].view(-1, Hq, d)[:, x].double() @ K.T * scale
                    s = s.masked_fill(torch.ones(s.shape, dtype=torch.bool).triu(len(keys) - m[b] + 1), -float("inf"))
                    p = torch.softmax(s, -1)
                    total += p.sum(0)
                    want = p @ V
                    # weights rounded to bf16 (2^-8 of each), the result too
                    tol = 2.0 ** -8 * (p @ V.abs() + want.abs()) + 1e-5
                    assert bool(((out.cpu()[t].view(-1, Hq, d)[:, x].double() - want).abs() <= tol).all()), (step, b, x)
                pg, row = table[b].long()[torch.arange(len(keys)) // page], torch.arange(len(keys)) % page
                have = before[pg, h, row].double()
                assert bool(((have - total).abs() <= 1e-4 * total + 1e-6).all()), (step, b, h)
                left = min(len(keys), 32)
                assert int(kv_len[b]) == left
                src = kept[b, h, :left].tolist()
                # the kernel's choice among its own weights
                order = sorted(range(2, len(keys) - 8), key=lambda j: (float(have[j]), -j), reverse=True)
                assert src == (sorted([0, 1] + list(range(len(keys) - 8, len(keys))) + order[:22]) if len(keys) > 32 else list(range(left)))
                model[b][h] = [keys[j] for j in src], [values[j] for j in src]
                gathered[b][h] = have[src]


def test_a_graph_of_weights_and_eviction_replays():
    c = U.make([1, 1], [300, 120], 4, 2, 64, 16, "bf16", seed=3, four=False)
    kp, vp = (A.pool_to_gpu(x, c.order) for x in (c.k_pool, c.v_pool))
    cache = A.cache_of(c, kp)
    q, lse = A.to_gpu(c.q), A.reference(c, 0.1, True)[1].float().cuda()
    w, e = old_weights(c).cuda(), D.make_eviction(budget=60, recent=4)
    w_out, left = torch.zeros_like(w), torch.zeros(2, dtype=torch.int32, device="cuda")
    kept = torch.zeros((2, 2, 60), dtype=torch.int32, device="cuda")
    ws, ws2 = D.alloc_attend_weights_workspace(cache), D.alloc_evict_workspace(cache, e)

    def step():
        D.dart_attend_weights(cache, q, kp, lse, w, ws, scale=0.1)
        D.dart_evict(cache, e, kp, vp, w, left, ws2, weights_out=w_out, kept=kept)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2, 3):
        results = []
        for go in (graph.replay, step):
            kp.copy_(c.k_pool)
            vp.copy_(c.v_pool)
            w.copy_(old_weights(c, seed))
            w_out.zero_()
            go()
            torch.cuda.synchronize()
            results.append([t.clone() for t in (kp, vp, w, w_out, left, kept)])
        for x, y in zip(*results):
            assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
