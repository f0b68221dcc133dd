"""What the calls on 4-bit pages, gathered weights and eviction do with page tables, scales and numbers that are out of the
ordinary: checks that run on the GPU (test_gpu_more_odd) and over the kernels' sources on the CPU (test_more_lanes_odd).
Their argument makes a call: more_gpu's or lanes_more_util's."""
import torch

import attend_util as A
import more_util as U


def bad_pages_of_evicted_keys(evict):
    """A page that is none is flagged wherever a key lies in it, and the other sequences are cut as always."""
    for four in (False, True):
        c = U.make([0] * 3, [100, 200, 90], 2, 2, 64, 16, "bf16", seed=1, four=four)
        w = torch.rand((c.k_pool.shape[0], 2, 16), generator=torch.Generator().manual_seed(2))
        before = c.four if four else (c.k_pool, c.v_pool)
        # (the first 16 keys lie in page 0, the recent 20 of 100 in pages 5 and 6; a sequence of 100 keeps all with the second)
        for how in (dict(budget=60, first=16, recent=20), dict(budget=100), dict(ratio=(1, 1))):
            good = evict(c, w, **how)
            assert good[4] == 0
            U.check_evicted(c, good[:4], w, **how)
            for place, page in ((0, -1), (3, 1 << 30), (5, c.k_pool.shape[0]), (6, -2 ** 31)):
                table = c.table.clone()
                table[0, place] = page
                pools, w_out, kept, left, status = evict(c, w, table=table, **how)
                assert status == 2, (how, place)
                assert torch.equal(left, good[3])
                for b in (1, 2):
                    at, row = U.places(c, b, int(left[b]))
                    for x, y in zip((pools[0], pools[1], (w_out,)), (good[0][0], good[0][1], (good[1],))):
                        for s, t in zip(x if isinstance(x, tuple) else (x,), y if isinstance(y, tuple) else (y,)):
                            assert torch.equal(s[at, :, row].contiguous().view(torch.uint8), t[at, :, row].contiguous().view(torch.uint8))
                    assert torch.equal(kept[b], good[2][b])
                # (what the page's number stood for before is nobody's key now: not read, not written)
                for x, y in zip(pools, before):
                    for s, t in zip(x if isinstance(x, tuple) else (x,), y if isinstance(y, tuple) else (y,)):
                        at = int(c.table[0, place])
                        assert torch.equal(s[at].contiguous().view(torch.uint8), t[at].contiguous().view(torch.uint8))
            table = c.table.clone()
            table[0, 7:] = -3  # behind the keys: not looked at
            table[2, 6:] = 1 << 30
            assert evict(c, w, table=table, **how)[4] == 0


def put_block(pool, page, head, row, block, scale, codes):
    """Scale and 32 codes of one block of a pool."""
    pool[1][page, head, row, block] = scale
    pool[0][page, head, row, 16 * block:16 * block + 16] = codes[::2] + 16 * codes[1::2]


def scales_that_no_append_writes_read(read):
    """Scale bytes 253 and 254 are read as their products, which the largest codes take beyond the type."""
    for dtype in ("bf16", "f32"):
        c = U.make([3], [3], 1, 1, 32, 16, dtype, seed=1)
        page, row = U.places(c, 0)
        codes = torch.arange(32, dtype=torch.uint8) % 16
        for t, scale in enumerate((252, 253, 254)):
            for pool in c.four:
                put_block(pool, page[t], 0, row[t], 0, scale, codes)
        want = torch.stack([U.GRID[codes.long() & 7] * torch.where(codes > 7, -1.0, 1.0) * 2.0 ** (e - 127) for e in (252, 253, 254)])
        for got in read(c)[:2]:
            assert torch.equal(got, want.to(c.dtype))
            assert torch.isinf(got.float()).sum(1).tolist() == [0, 8, 16]


def scales_that_no_append_writes_attend(attend):
    """Values of such a block, infinite and finite, go to the rows that see their key, and to no others."""
    for dtype in ("bf16", "f32"):
        # many rows; few, in pages that hold whole tiles and in smaller ones; wide heads
        for n, d, page in (([70, 1], 96, 16), ([6], 96, 16), ([6], 96, 4), ([6], 256, 16), ([70], 256, 16)):
            for scale in (253, 254):
                c = U.make(n, [130, 40][:len(n)], 4, 2, d, page, dtype, seed=9)
                at, row = U.places(c, 0)
                key = 126  # seen by the last four tokens of the first sequence
                # codes of 0, of 2^(scale - 128) and of what is infinite
                codes = torch.tensor([0, 1, 9, 7], dtype=torch.uint8).repeat(8)
                put_block(c.four[1], at[key], 1, row[key], 1, scale, codes)
                c.v_pool[at[key], 1, row[key], 32:64] = torch.tensor([0.0, 0.5, -0.5, 0.0], dtype=torch.float64).repeat(8) * 2.0 ** (scale - 127)
                # (scores so near one another that weights of the running reference do not carry the finite ones out of range)
                want, want_lse, tol, lse_tol = A.reference(c, 0.02, True)
                out, lse, status = attend(c, scale=0.02)[:3]
                assert status == 0
                spoilt = torch.zeros(out.shape, dtype=torch.bool)
                spoilt[n[0] - 4:n[0], 2:, 35:64:4] = True
                assert bool((out[spoilt] == float("inf")).all()), (dtype, n, d, page, scale)
                assert bool(((out.double() - want).abs() <= tol)[~spoilt].all()), (dtype, n, d, page, scale)
                assert bool(((lse.double() - want_lse).abs() <= lse_tol).all())


def many_rows(dtype, four, join=False, **more):
    """A case whose rows gathered weights take by tiles of many (over 48 of a sequence); join: in several parts."""
    n, kv = ([1, 300, 6], [50, 420, 6]) if join else ([1, 90, 6], [90, 150, 2])
    return U.make(n, kv, 4, 2 if not join else 1, 64, 16, dtype, seed=6, four=four, **more)


def old_weights(c):
    return torch.rand((c.k_pool.shape[0], c.k_pool.shape[1], c.page), generator=torch.Generator().manual_seed(3))


def weights_of_many_rows(weights):
    """Scales of either sign and none, rows that see nothing, numbers that are none, skipped sequences: by the tiles of many rows,
    in one part and in several."""
    inf, nan = float("inf"), float("nan")
    for dtype in ("bf16", "f32"):
        for four in (False, True):
            for join in (False, True):
                where = (dtype, four, join)
                c = many_rows(dtype, four, join)
                old = old_weights(c)
                for scale in (-0.3, 0.0, 1.0):
                    for causal in (True, False):
                        lse = A.reference(c, scale, causal)[1].float()
                        got, status = weights(c, lse, old, scale=scale, causal=causal, carry=0.5)[:2]
                        assert status == 0
                        U.check_gathered(c, got, lse, old, scale=scale, causal=causal, carry=0.5)

                # lse that is no number: -inf gives nothing, +inf neither, NaN goes to the keys that the row sees
                scale = 0.1
                lse = A.reference(c, scale, True)[1].float()
                t, last = int(c.cu[1]) + 20, c.kv[1] - c.n[1] + 20  # a token of the second sequence, the last key it sees
                good = weights(c, lse, old, scale=scale)[0]
                one = lse.clone()
                one[t, 1] = -inf
                none = weights(c, one, old, scale=scale)[0]
                U.check_gathered(c, none, one, old, scale=scale, causal=True, carry=1.0)
                one[t, 1] = inf  # (exp(s - inf) = 0; no finite error can be derived from such an lse)
                assert torch.equal(weights(c, one, old, scale=scale)[0], none), where
                one[t, 1] = nan
                got = weights(c, one, old, scale=scale)[0]
                page, row = U.places(c, 1)
                spoilt = torch.zeros(got.shape, dtype=torch.bool)
                spoilt[page[:last + 1], 0, row[:last + 1]] = True
                assert torch.isnan(got[spoilt]).all() and torch.equal(got[~spoilt], good[~spoilt]), where

                # keys that are none spoil their own weight, whether all rows of a tile see them or some
                d = many_rows(dtype, four, join)
                spoilt = torch.zeros(got.shape, dtype=torch.bool)
                for key in (5, c.kv[1] - c.n[1] + 70, c.kv[1] - 1):
                    at = int(page[key]), 0, int(row[key])
                    spoilt[at] = True
                    if four:
                        d.four[0][1][(*at, 1)] = 255
                    else:
                        d.k_pool[(*at, 33)] = nan
                got = weights(d, lse, old, scale=scale)[0]
                assert torch.isnan(got[spoilt]).all() and torch.equal(got[~spoilt], good[~spoilt]), where

                # a sequence that is skipped keeps its weights, a key whose page is none has none; the others are as always
                kv = torch.tensor(c.kv, dtype=torch.int32)
                kv[1] = -4
                got, status = weights(c, lse, old, scale=scale, kv=kv)[:2]
                assert status == 1 and torch.equal(got[page, :, row], old[page, :, row])
                for b in (0, 2):
                    at, r = U.places(c, b)
                    assert torch.equal(got[at, :, r], good[at, :, r]), where
                table = c.table.clone()
                table[1, 2] = 1 << 29
                got, status = weights(c, lse, old, scale=scale, table=table)[:2]
                keys = torch.arange(c.kv[1])
                lost = (keys >= 32) & (keys < 48)
                assert status == 2 and torch.equal(got[page[~lost], :, row[~lost]], good[page[~lost], :, row[~lost]]), where
                assert torch.equal(got[page[lost], :, row[lost]], old[page[lost], :, row[lost]]), where


def weights_of_prefixes_of_many_rows(weights):
    """A group with a skipped sequence is skipped whole; the other one is as always."""
    for dtype in ("bf16", "f32"):
        for four in (False, True):
            c = U.make([80, 3, 120], [85, 20, 130], 4, 2, 64, 16, dtype, groups=[2, 1], prefix=[200, 300], seed=6, four=four)
            lse, old = A.reference(c, -0.1, True)[1].float(), old_weights(c)
            good, status = weights(c, lse, old, scale=-0.1, carry=0.25)[:2]
            assert status == 0
            U.check_gathered(c, good, lse, old, scale=-0.1, causal=True, carry=0.25)
            kv = torch.tensor(c.kv, dtype=torch.int32)
            kv[1] = 1 << 20
            got, status = weights(c, lse, old, scale=-0.1, carry=0.25, kv=kv)[:2]
            assert status == 1
            for places, same in ((U.places(c, 0), good), (U.places(c, 1), old), (U.places(c, 2), good),
                                 (U.places(c, None, 200, c.front[0]), old), (U.places(c, None, 300, c.front[1]), good)):
                assert torch.equal(got[places[0], :, places[1]], same[places[0], :, places[1]])
