"""Token offsets that hold anything at all: their sequences are skipped and flagged, the others are as they were."""
import pytest
import torch

import paper_2502_11494_amd as D

import attend_util as A

pytestmark = pytest.mark.gpu

LEAST, MOST = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("sequences", [4, 70])  # (looked up in one go, and by searches)
@pytest.mark.parametrize("value", [LEAST, LEAST + 5, -1, MOST])
def test_offsets_at_the_ends_of_their_type(sequences, value):
    n = [2, 3, 4, 5] + [1] * (sequences - 4)
    c = A.make(n, [50 + x for x in n], 4, 2, 64, 16, "bf16", seed=10)
    want = A.attend(c, scale=0.1)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cu = c.cu.clone()
    cu[sequences] = value  # the end of the last sequence: nothing before it is touched
    out, lse = A.attend(c, scale=0.1, status=status, cu=cu)
    assert int(status) == 1
    last = int(c.cu[sequences - 1])
    assert torch.equal(out[:last], want[0][:last]) and torch.equal(lse[:last], want[1][:last])
    pool = torch.full((8, 4, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    rows = torch.ones((c.T, 4 * 64), dtype=torch.bfloat16, device="cuda")
    table = torch.arange(sequences, dtype=torch.int32, device="cuda").view(-1, 1) % 8
    kv = torch.tensor(n, dtype=torch.int32, device="cuda").clamp(max=4)
    cache = D.make_cache(4, pool, table, kv, 4, T=c.T, cu_q=cu.cuda())
    k_pool, v_pool = pool.clone(), pool.clone()
    status.zero_()
    r = D.make_rotation(4, 4, 64, D.DART_BF16, torch.ones(32, device="cuda"))
    D.dart_norm_rotate_append(r, cache, rows, rows, rows, torch.zeros(c.T, dtype=torch.int64, device="cuda"), torch.empty_like(rows), k_pool,
                              v_pool, status=status)
    torch.cuda.synchronize()
    assert int(status) == 1
    for p in (k_pool, v_pool):
        assert bool(((p == 1.0) | (p == 3.0)).all())
