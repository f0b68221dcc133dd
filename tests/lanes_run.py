"""The kernels on the CPU between guard pages (lanes_util), a group of cases at a time: an access out of bounds ends this
process, so the tests start it as one of their own.

    python tests/lanes_run.py tiles | widest | prefixes | joins | garbage | rows
"""
import faulthandler
import os
import random
import sys

sys.path[:0] = [os.path.dirname(os.path.abspath(__file__)), os.path.dirname(os.path.dirname(os.path.abspath(__file__)))]
import torch  # noqa: E402

import attend_util as A  # noqa: E402
import lanes_util as L  # noqa: E402
import paper_2502_11494_amd as D  # noqa: E402


def kinds(launches):
    """(type, width, columns, waves of rows, key groups) of the tile kernels among the launches, "both" and "join" beside."""
    found = set()
    for line in launches.splitlines():
        if "launch_tiles" in line:
            v = dict(x.strip().split(" = ") for x in line[line.rindex("[") + 1:line.rindex("]")].split(","))
            found.add(("f32", "bf16")[int(v["DT"])] + " " + " ".join(v[k] for k in ("DP", "QW", "WM", "WK")))
        elif "launch_both" in line:
            v = dict(x.strip().split(" = ") for x in line[line.rindex("[") + 1:line.rindex("]")].split(","))
            found.add("both " + ("f32", "bf16")[int(v["DT"])] + " " + v["DP"])
        elif "dart_attend" in line:
            found.add("join")
    return found


def run(c, name, *, scale=0.11, causal=True, sides=2, expect=(), **how):
    """The same in both orders of lanes (or one of them), buffers against the guard page behind them and against the one in front."""
    first = None
    for at_end, back in ((True, False), (False, True)) if sides == 2 else ((bool(sides), not sides),):
        out, lse, status, launches = L.attend(c, scale=scale, causal=causal, at_end=at_end, back=back, **how)
        assert status == 0, status
        A.check(c, (out, lse), scale=scale, causal=causal)
        assert first is None or (torch.equal(out, first[0]) and torch.equal(lse, first[1])), "the order of lanes shows"
        first = first or (out, lse)
    got = kinds(launches)
    assert set(expect) <= got, (expect, got)
    print(name, sorted(got), flush=True)


N, KV = [1, 0, 3, 17, 1, 64, 33, 5, 1, 30], [1, 9, 3, 40, 0, 65, 20, 128, 300, 157]


def tiles():
    for dtype in ("bf16", "f32"):
        for d in (8, 40, 64, 80, 96, 128, 192, 256):
            dp = 64 if d <= 64 else 128 if d <= 128 else 256
            few = f"{dtype} {dp} 16 4 1" if dtype == "f32" and dp == 256 else f"{dtype} {dp} 16 1 4"
            many = f"{dtype} {dp} {32 if dtype == 'bf16' and dp <= 128 else 16} 4 1"
            for causal in (True, False):
                run(A.make(N, KV, 12, 4, d, 16, dtype, seed=d), f"prompts {dtype} {d}", causal=causal, expect=[many])
                run(A.make([1, 0, 3, 2], [1, 9, 3, 40], 4, 2, d, 4, dtype, seed=d), f"few {dtype} {d}", causal=causal, expect=[few])
            run(A.make([1] * 6, [1, 2, 33, 0, 129, 600], 8, 2, d, 16, dtype, "rows", seed=d), f"single {dtype} {d}", expect=[few])
            run(A.make([1, 2], [700, 1100], 40, 1, d, 32, dtype, seed=d), f"long {dtype} {d}", expect=["join"])
    for page in (1, 2, 64, 2048):
        run(A.make([1, 20, 7], [77, 20, 200], 6, 3, 64, page, "bf16", seed=page), f"pages of {page}", ld=3)


def widest():
    n = [129, 300, 1, 0, 256, 257, 140, 133, 200, 180, 255, 90, 300, 31, 280, 256, 290]
    kv = [130, 300, 9, 5, 40, 257, 0, 150, 200, 181, 255, 90, 310, 31, 280, 256, 290]
    for d, dp, causal in ((64, 64, True), (128, 128, False)):
        c = A.make(n, kv, 32, 32, d, 32, "bf16", seed=d)
        assert c.T // 256 * 32 >= 384
        run(c, f"own {d}", max_kv=1024, causal=causal, sides=int(causal), expect=[f"bf16 {dp} 32 8 1"])
    # prefixes in the widest tiles, own keys in them and not
    kv = [a + a % 3 for a in n]
    c = A.make(n, kv, 32, 32, 64, 32, "bf16", groups=[5, 0, 8, 4], prefix=[70, 9, 0, 129], seed=1)
    run(c, "prefixes", max_prefix=1024, max_kv=1024, sides=1, expect=["bf16 64 32 8 1", "join"])
    c = A.make(n, kv, 32, 32, 96, 32, "bf16", groups=[17], prefix=[65], seed=2)
    run(c, "one prefix", max_prefix=2000, sides=0, expect=["bf16 128 32 8 1", "join"])


def prefixes():
    n, kv = [5, 1, 0, 33, 2, 1, 30, 1, 8], [5, 4, 64, 133, 19, 1, 61, 251, 17]
    for dtype in ("bf16", "f32"):
        for d in (40, 64, 80, 96, 128, 256):
            dp = 64 if d <= 64 else 128 if d <= 128 else 256
            expect = [f"both {dtype} {dp}", "join"] if dtype == "bf16" or dp <= 128 else [f"f32 {dp} 16 4 1", "join"]
            for causal in (True, False):
                run(A.make(n, kv, 4, 2, d, 16, dtype, groups=[4, 0, 2, 3], prefix=[70, 5, 0, 600], seed=d), f"prompts {dtype} {d}",
                    causal=causal, expect=expect, ld=5)
            run(A.make([1] * 9, [max(1, x) for x in kv], 14, 2, d, 16, dtype, groups=[9], prefix=[333], seed=d), f"steps {dtype} {d}",
                expect=expect)
    run(A.make([40, 33, 1, 50] * 4, [45, 33, 9, 60] * 4, 32, 32, 64, 32, "f32", groups=[9, 7], prefix=[90, 0], seed=4), "two launches",
        expect=["f32 64 16 4 1", "join"])


def joins():
    n = [i % 3 for i in range(72)]
    kv = [a + i * 53 % 300 for i, a in enumerate(n)]
    run(A.make(n, kv, 4, 1, 64, 16, "bf16", seed=72), "searches", max_kv=700)
    groups = [1] * 60 + [2] * 6
    run(A.make(n, kv, 4, 2, 64, 16, "bf16", groups=groups, prefix=[i * 37 % 90 for i in range(66)], seed=73), "searches of groups",
        expect=["join"])
    run(A.make([1] * 72, [1 + x for x in kv], 4, 1, 40, 16, "f32", groups=groups, prefix=[i * 37 % 90 for i in range(66)], seed=74),
        "searches of single tokens", expect=["join"])


def garbage():
    """Device arrays that hold anything: nothing is read or written out of bounds, and what is wrong is flagged."""
    rnd = random.Random(1)
    ints = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    flagged = 0
    for i in range(160):
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
        c = A.make(n, kv, r * Hkv, Hkv, d, rnd.choice((1, 4, 16)), dtype, groups=groups,
                   prefix=[rnd.choice((0, 1, 40, 90)) for _ in groups] if groups else None, seed=i)
        wild = (-2 ** 31, -1, 0, 1, 3, 100, 2 ** 31 - 1)

        def spoil(v, low, high, much):
            return ints([x if rnd.random() > much else rnd.choice(wild) if rnd.random() < 0.3 else rnd.randint(low, high) for x in v])

        much = rnd.choice((0.1, 0.5, 1.0))
        how = dict(cu=spoil(c.cu.tolist(), -3, c.T + 3, much), kv=spoil(kv, -2, 90, much), max_q=rnd.choice((None, 1, 3, c.T)),
                   max_kv=rnd.choice((None, 0, 10, 500)), packed=True, n_pages=rnd.choice((None, 1)), ld=rnd.choice((0, 2)),
                   table=spoil(c.table.flatten().tolist(), -1, c.k_pool.shape[0], much * 0.5).view(c.table.shape))
        if groups:
            how.update(group_cu=spoil([sum(groups[:j]) for j in range(len(groups) + 1)], -2, B + 2, much),
                       prefix=spoil(c.prefix, -2, 120, much).tolist(), max_prefix=rnd.choice((None, 0, 500)))
            c.front = spoil(c.front.flatten().tolist(), -1, c.k_pool.shape[0], much * 0.5).view(c.front.shape)
        for at_end in (True, False):
            status = L.attend(c, scale=0.1, causal=rnd.random() < 0.7, at_end=at_end, back=not at_end, **how)[2]
            assert status & ~3 == 0
            flagged += status != 0
        for key in ("group_cu", "prefix", "max_prefix"):
            how.pop(key, None)
        q, k = (torch.randn((c.T, h * 64)).to(c.dtype) for h in (8, 8))
        c8 = A.make(n, kv, 8, 8, 64, 4, dtype, seed=i)
        how["table"] = spoil(c8.table.flatten().tolist(), -1, c8.k_pool.shape[0], much * 0.5).view(c8.table.shape)
        status = L.append(c8, rotation(8, 8, 64, c8.dtype, 32), q, k, k, torch.arange(c.T), at_end=i % 2 == 0, **how)[4]
        assert status & ~3 == 0
        flagged += status != 0
        print(i, B, c.T, r, Hkv, d, dtype, flush=True)
    assert flagged > 100


def rotation(Hq, Hkv, d, dtype, half, weights=None, interleaved=0):
    """What makes the descriptor, its arrays between guard pages."""
    def make(buf):
        r = D.DartRotation()
        r.Hq, r.Hkv, r.d, r.dtype, r.rot, r.interleaved, r.planes, r.eps, r.scale = (Hq, Hkv, d, A.KIND[dtype], 2 * half, interleaved, 1,
                                                                                      1e-6, 1.0)
        r.inv_freq = buf.copy(10000.0 ** (-torch.arange(half, dtype=torch.float32) / max(half, 1)))
        if weights is not None:
            r.q_weight = r.k_weight = buf.copy(weights)
        return r
    return make


def rows():
    """Rotation and append.  (Head counts of which whole rounds of lanes are queries, keys or values.)"""
    from test_gpu_norm_rotate import definition, within
    for dtype in ("bf16", "f32"):
        for H, d, rot in ((8, 64, 64), (16, 128, 128), (16, 80, 40), (8, 256, 64), (32, 40, 8), (64, 8, 8), (32, 64, 0)):
            for n, kv, page in (([1, 1, 1], [5, 16, 33], 16), ([3, 0, 9, 1], [3, 7, 40, 17], 4), ([600, 500], [600, 700], 64)):
                if sum(n) > 1000 and H * d > 600:
                    continue
                c = A.make(n, kv, H, H, d, page, dtype, seed=d, order="rows" if page == 4 else "heads")
                g = torch.Generator().manual_seed(rot)
                q, k, v = (torch.randn((c.T, H * d), generator=g).to(c.dtype) for _ in range(3))
                pos, weight = torch.randint(0, 9000, (c.T,), generator=g), (torch.rand(d, generator=g) + 0.5).to(c.dtype)
                freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float32) / max(rot // 2, 1))
                for at_end, back in ((True, False), (False, True)):
                    for inter in (0, 1):
                        got = L.append(c, rotation(H, H, d, c.dtype, rot // 2, weight, inter), q, k, v, pos, at_end=at_end, back=back, ld=2)
                        assert got[4] == 0
                        want, tol = definition(q, H, d, rot, pos[None], [rot // 2], freq, inter, weight, 1.0)
                        within(got[0].view(c.T, H, d), want, tol, c.dtype)
                        want, tol = definition(k, H, d, rot, pos[None], [rot // 2], freq, inter, weight, 1.0)
                        pools = c.k_pool.clone(), c.v_pool.clone()
                        for b, m in enumerate(n):
                            at = torch.arange(kv[b] - m, kv[b])
                            t = torch.arange(int(c.cu[b]), int(c.cu[b + 1]))
                            page_of, row = c.table[b].long()[at // page], at % page
                            if m:
                                within(got[1][page_of, :, row].reshape(m, H, d), want[t], tol[t], c.dtype)
                            pools[0][page_of, :, row] = got[1][page_of, :, row]
                            pools[1][page_of, :, row] = v.view(c.T, H, d)[t]
                        for have, should in zip(got[1:3], pools):  # (rows of no token are left alone, NaN bits and all)
                            assert torch.equal(have.contiguous().view(torch.uint8), should.contiguous().view(torch.uint8))
                print(dtype, H, d, rot, n, flush=True)


if __name__ == "__main__":
    faulthandler.enable()
    torch.set_num_threads(1)
    globals()[sys.argv[1]]()
    print("lanes ok", flush=True)
