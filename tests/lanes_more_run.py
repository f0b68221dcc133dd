"""The kernels on 4-bit pages, gathered weights and eviction on the CPU between guard pages (lanes_more_util), a group of cases at
a time: an access out of bounds ends this process, so the tests start it as one of their own.

    python tests/lanes_more_run.py hold | attend | share | weights | prefixes | evict | garbage
"""
import faulthandler
import os
import random
import sys

sys.path[:0] = [os.path.dirname(os.path.abspath(__file__)), os.path.dirname(os.path.dirname(os.path.abspath(__file__)))]
import torch  # noqa: E402

import attend_util as A  # noqa: E402
import lanes_more_util as M  # noqa: E402
import more_util as U  # noqa: E402

N, KV = [1, 0, 3, 17, 1, 64, 33, 5, 1, 30], [1, 9, 3, 40, 0, 65, 20, 128, 300, 157]
SIDES = ((True, False), (False, True))


def same(x, y):
    return torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


def hold():
    """Append and read: the format's definition, rows of no token left alone."""
    g = torch.Generator().manual_seed(0)
    for dtype in ("bf16", "f32"):
        for Hkv, d, page, order in ((2, 8, 16, "heads"), (3, 40, 4, "rows"), (2, 64, 1, "heads"), (2, 96, 64, "rows"), (1, 256, 16, "heads"),
                                    (20, 80, 16, "heads")):
            c = U.make([1, 3, 0, 20, 2], [5, 40, 3, 33, 1], Hkv, Hkv, d, page, dtype, order, seed=d)
            k, v = ((torch.randn((c.T, Hkv * d), generator=g) * torch.exp(4 * torch.randn((c.T, Hkv * d), generator=g))).to(c.dtype) for _ in range(2))
            for at_end, back in SIDES:
                kp, vp, status = M.append(c, k, v, at_end=at_end, back=back, ld=3)
                assert status == 1  # (the last sequence has more tokens than keys)
                for have, before, x in ((kp, c.four[0], k), (vp, c.four[1], v)):
                    want, packed = tuple(t.clone() for t in before), U.pack(x.view(c.T, Hkv, d))
                    for b, n in enumerate(c.n[:4]):
                        if n:
                            pg, row = (t[-n:] for t in U.places(c, b))
                            for w, p in zip(want, packed):
                                w[pg, :, row] = p[int(c.cu[b]):int(c.cu[b + 1])]
                    assert all(torch.equal(a, w) for a, w in zip(have, want)), (dtype, d)
                held = c.four
                c.four = kp, vp
                for x, out in zip((k, v), M.read(c, at_end=at_end, back=back)[:2]):
                    want = U.unpack(U.pack(x.view(c.T, Hkv, d)), d).reshape(c.T, -1)
                    want[-2:] = 7.0
                    assert torch.equal(out.double(), want), (dtype, d)
                c.four = held
            print("hold", dtype, d, flush=True)


def run(c, name, scale=0.11, causal=True, **how):
    first = None
    for at_end, back in SIDES:
        out, lse, status, launches = M.attend(c, scale=scale, causal=causal, at_end=at_end, back=back, **how)
        assert status == 0, status
        A.check(c, (out, lse), scale=scale, causal=causal)
        assert first is None or (same(out, first[0]) and same(lse, first[1])), "the order of lanes shows"
        first = first or (out, lse)
    print(name, launches.count("\n"), flush=True)
    return launches


def attend():
    for dtype in ("bf16", "f32"):
        for d in (8, 64, 80, 128, 256):
            for causal in (True, False):
                run(U.make(N, KV, 12, 4, d, 16, dtype, seed=d), f"prompts {dtype} {d}", causal=causal)
                run(U.make([1, 0, 3, 2], [1, 9, 3, 40], 4, 2, d, 4, dtype, seed=d), f"few, small pages {dtype} {d}", causal=causal)
                run(U.make([1, 0, 3, 2], [1, 9, 3, 140], 4, 2, d, 64, dtype, "rows", seed=d), f"few {dtype} {d}", causal=causal, ld=3)
            run(U.make([1] * 6, [1, 2, 33, 0, 129, 600], 8, 2, d, 16, dtype, "rows", seed=d), f"single {dtype} {d}")
            run(U.make([1, 2], [700, 1100], 40, 1, d, 32, dtype, seed=d), f"long {dtype} {d}")
    n = [129, 300, 1, 0, 256, 257, 140, 133, 200, 180, 255, 90, 300, 31, 280, 256, 290]
    run(U.make(n, [a + a % 3 for a in n], 32, 32, 64, 32, "bf16", seed=1), "widest", max_kv=1024)


def share():
    """Parts cut on the device for what all sequences hold together; bounds far above the lengths."""
    for dtype, d in (("bf16", 64), ("bf16", 128), ("f32", 64)):
        c = U.make([1, 1, 1, 1, 1], [1500, 3, 0, 700, 40], 4, 1, d, 16, dtype, seed=d)
        for max_kv in (1500, 20000):
            launches = run(c, f"share {dtype} {d} {max_kv}", max_kv=max_kv)
            assert "join" in launches
        run(U.make([2, 0, 1, 3], [1500, 3, 1, 700], 4, 1, d, 32, dtype, seed=d), f"share, packed {dtype} {d}", max_kv=3000, ld=2)
    # a bound as far as it goes: many parts that no sequence has, their numbers times the keys of one beyond 32 bits
    run(U.make([1, 1], [9000, 2000], 1, 1, 8, 16, "bf16", seed=5), "share, far bound", max_kv=2 ** 22)


def weigh(c, name, scale=0.11, causal=True, carry=0.5, **how):
    lse = A.reference(c, scale, causal)[1].float()
    pages, Hkv = c.k_pool.shape[:2]
    old, first = torch.rand((pages, Hkv, c.page)), None
    for at_end, back in SIDES:
        got, status, launches = M.weights(c, lse, old, scale=scale, causal=causal, carry=carry, at_end=at_end, back=back, **how)
        assert status == 0
        U.check_gathered(c, got, lse, old, scale=scale, causal=causal, carry=carry)
        assert first is None or same(got, first), "the order of lanes shows"
        first = got
    print(name, launches.count("\n"), flush=True)
    return launches


def weights():
    for four in (False, True):
        for dtype in ("bf16", "f32"):
            for d in (8, 64, 80, 128, 256):
                for causal in (True, False):
                    weigh(U.make([1, 0, 3, 17, 1, 64, 30], [1, 9, 3, 40, 0, 400, 157], 12, 4, d, 16, dtype, seed=d, four=four),
                          f"prompts {four} {dtype} {d}", causal=causal, carry=float(causal))
                weigh(U.make([1] * 5, [1, 300, 33, 0, 129], 8, 2, d, 1 if d == 8 else 16, dtype, "rows", seed=d, four=four),
                      f"single {four} {dtype} {d}", ld=2)
            launches = weigh(U.make([200, 3], [230, 300], 4, 1, 64, 64, dtype, seed=3, four=four), f"parts {four} {dtype}", carry=0.0)
            assert "k_join" in launches or launches.count("\n") == 2


def prefixes():
    n, kv = [5, 1, 0, 33, 2, 1, 30, 1, 8], [5, 4, 64, 133, 19, 1, 61, 251, 17]
    for dtype in ("bf16", "f32"):
        for d in (40, 80, 128, 256):
            for four in (False, True):
                c = U.make(n, kv, 4, 2, d, 16, dtype, groups=[4, 0, 2, 3], prefix=[70, 5, 0, 600], seed=d, four=four)
                weigh(c, f"weights {four} {dtype} {d}", ld=3)
            run(c, f"attend {dtype} {d}", ld=5)
            run(U.make([1] * 9, [max(1, x) for x in kv], 14, 2, d, 16, dtype, groups=[9], prefix=[333], seed=d), f"steps {dtype} {d}")
    weigh(U.make([90, 0, 150], [90, 5, 160], 4, 1, 64, 16, "bf16", groups=[2, 1], prefix=[300, 20], seed=1), "parts of prefixes")


def evict():
    g = torch.Generator().manual_seed(1)
    for four in (False, True):
        for dtype in ("bf16", "f32"):
            for Hkv, d, page, order in ((2, 8, 1, "heads"), (2, 40, 16, "rows"), (1, 128, 64, "heads"), (2, 96, 256, "rows"), (2, 256, 4, "heads")):
                c = U.make([0] * 5, [0, 3, 200, 130, 500], Hkv, Hkv, d, page, dtype, order, seed=d, four=four)
                w = torch.randn((c.k_pool.shape[0], Hkv, page), generator=g)
                w = w.round() if d == 40 else torch.ones_like(w) if d == 8 else w
                for how in (dict(budget=129, first=1, recent=2), dict(ratio=(3, 10)), dict(budget=5, recent=9)):
                    for (at_end, back), (out, keep) in zip(SIDES, (("other", True), ("same", False))):
                        got = M.evict(c, w, out=out, keep=keep, at_end=at_end, back=back, ld=2, packed=True, **how)
                        assert got[4] == 0
                        U.check_evicted(c, got[:4], w, **how)
                got = M.evict(c, w, out=None, packed=True, budget=50)
                U.check_evicted(c, got[:4], w, budget=50)
                print("evict", four, dtype, d, flush=True)
    for n, kind in ((3000, 0), (17000, 0), (17000, 1), (33000, 2)):  # every kernel, and sequences that it reads again by every step
        c = U.make([0, 0], [n, 700], 1, 1, 8, 256, "bf16", seed=n, four=False)
        w = torch.randn((c.k_pool.shape[0], 1, 256), generator=g)
        w = w if kind == 0 else w.round() if kind == 1 else torch.zeros_like(w)
        for how in (dict(budget=1500), dict(ratio=(9, 10), first=4, recent=100)):
            got = M.evict(c, w, packed=True, **how)
            U.check_evicted(c, got[:4], w, **how)
        print("evict", n, kind, flush=True)


def garbage():
    """Device arrays that hold anything: nothing is read or written out of bounds, and what is wrong is flagged."""
    rnd = random.Random(1)
    ints = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    flagged = 0
    for i in range(110):
        B = rnd.choice((1, 2, 5, 9, 70))
        n = [rnd.choice((0, 1, 1, 2, 7, 40)) for _ in range(B)]
        if sum(n) == 0:
            n[0] = 1
        kv = [rnd.choice((0, 1, 5, 20, 70)) for _ in range(B)]
        r, Hkv, d, dtype = rnd.choice((1, 2, 7)), rnd.choice((1, 2)), rnd.choice((8, 64, 80, 256)), rnd.choice(("bf16", "f32"))
        groups = None
        if rnd.random() < 0.5:
            groups = [0] * rnd.randint(1, B)
            for _ in range(B):
                groups[rnd.randrange(len(groups))] += 1
        c = U.make(n, kv, r * Hkv, Hkv, d, rnd.choice((1, 4, 16)), dtype, groups=groups,
                   prefix=[rnd.choice((0, 1, 40, 90)) for _ in groups] if groups else None, seed=i, four=rnd.random() < 0.7)
        wild = (-2 ** 31, -1, 0, 1, 3, 100, 2 ** 31 - 1)

        def spoil(v, low, high, much):
            return ints([x if rnd.random() > much else rnd.choice(wild) if rnd.random() < 0.3 else rnd.randint(low, high) for x in v])

        much = rnd.choice((0.1, 0.5, 1.0))
        how = dict(cu=spoil(c.cu.tolist(), -3, c.T + 3, much), kv=spoil(kv, -2, 90, much), max_q=rnd.choice((None, 1, 3, c.T)),
                   max_kv=rnd.choice((None, 0, 10, 500, 3000)), packed=True, n_pages=rnd.choice((None, 1)), ld=rnd.choice((0, 2)),
                   table=spoil(c.table.flatten().tolist(), -1, c.k_pool.shape[0], much * 0.5).view(c.table.shape))
        plain = dict(how)
        if groups:
            how.update(group_cu=spoil([sum(groups[:j]) for j in range(len(groups) + 1)], -2, B + 2, much),
                       prefix=spoil(c.prefix, -2, 120, much).tolist(), max_prefix=rnd.choice((None, 0, 500)))
            c.front = spoil(c.front.flatten().tolist(), -1, c.k_pool.shape[0], much * 0.5).view(c.front.shape)
        lse, old = torch.randn((c.T, c.Hq)), torch.rand((c.k_pool.shape[0], Hkv, c.page))
        lse[rnd.randrange(c.T)] = rnd.choice((float("nan"), float("inf"), -float("inf")))
        for at_end in (True, False):
            side = dict(at_end=at_end, back=not at_end)
            causal, statuses = rnd.random() < 0.7, []
            statuses.append(M.weights(c, lse, old, scale=0.1, causal=causal, **how, **side)[1])
            e = dict(budget=rnd.choice((0, 1, 7, 30)), ratio=(rnd.randint(0, 5), 5), first=rnd.choice((0, 2, 50)), recent=rnd.choice((0, 3)))
            statuses.append(M.evict(c, old, keep=at_end, out=rnd.choice(("other", "same", None)), **e, **plain, **side)[4])
            if c.four is not None:
                statuses.append(M.attend(c, scale=0.1, causal=causal, **how, **side)[2])
                k = torch.randn((c.T, Hkv * d)).to(c.dtype)
                statuses.append(M.append(c, k, k, **how, **side)[2])
                statuses.append(M.read(c, **how, **side)[2])
            assert all(s & ~3 == 0 for s in statuses), statuses
            flagged += any(statuses)
        print(i, B, c.T, r, Hkv, d, dtype, flush=True)
    assert flagged > 100


if __name__ == "__main__":
    faulthandler.enable()
    torch.set_num_threads(1)
    globals()[sys.argv[1]]()
    print("lanes ok", flush=True)
