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
