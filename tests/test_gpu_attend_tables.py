"""Page tables that are views of wider ones: their own entries are used, and none beside them."""
import pytest
import torch

import paper_2502_11494_amd as D

import attend_util as A

pytestmark = pytest.mark.gpu


def inside(table, before, after, decoys):
    """`table` as a view of a wider one; the entries around it name `decoys`, pages of the pool."""
    B, n = table.shape
    base = torch.empty((B, before + n + after), dtype=torch.int32)
    base[:] = torch.tensor(decoys, dtype=torch.int32)[torch.arange(base.numel()).view(base.shape) % len(decoys)]
    base[:, before:before + n] = table
    return base.cuda()[:, before:before + n]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("before,after", [(24, 0), (3, 5), (0, 1)])
def test_attention_through_a_view(dtype, before, after):
    c = A.make([1, 40, 3, 7], [77, 40, 500, 130], 6, 3, 64, 16, dtype, groups=[1, 3], prefix=[100, 33], seed=1)
    other = [int(c.table[1, 0])]
    k_pool, v_pool = c.k_pool.cuda(), c.v_pool.cuda()
    kv, cu = torch.tensor(c.kv, dtype=torch.int32).cuda(), c.cu.cuda()
    front = dict(group_cu=torch.tensor([0, 1, 4], dtype=torch.int32).cuda(), max_prefix=100,
                 prefix_len=torch.tensor(c.prefix, dtype=torch.int32).cuda())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(table, prefix, kv=kv, prefix_len=None, max_kv=500, max_prefix=100):
        more = dict(front, max_prefix=max_prefix)
        if prefix_len is not None:
            more["prefix_len"] = prefix_len
        cache = D.make_cache(6, k_pool, table, kv, max_kv, T=c.T, max_q=40, cu_q=cu, prefix_pages=prefix, **more)
        out, lse = torch.empty((c.T, 384), dtype=c.dtype, device="cuda"), torch.empty((c.T, 6), device="cuda")
        status.zero_()
        D.dart_attend(cache, A.to_gpu(c.q), k_pool, v_pool, out, D.alloc_attend_workspace(cache), scale=0.125, lse=lse,
                      status=status)
        torch.cuda.synchronize()
        return out.cpu().view(c.T, 6, 64), lse.cpu()

    table, prefix = inside(c.table, before, after, other), inside(c.front, before, after, other)
    good = run(table, prefix)
    assert int(status) == 0
    A.check(c, good, scale=0.125)
    # longer than the view has pages, though not than the table it is a view of
    more = 16 * c.table.shape[1] + 1
    long = kv.clone()
    long[3] = more
    out, lse = run(table, prefix, kv=long, max_kv=more)
    rows = slice(int(c.cu[3]), c.T)
    assert int(status) == 1
    assert bool((out[rows] == 0).all()) and bool((lse[rows] == -float("inf")).all())
    tol = A.reference(c, 0.125, True)
    assert bool(((out.double() - tol[0]).abs() <= tol[2])[:rows.start].all())
    more = 16 * c.front.shape[1] + 1
    out, lse = run(table, prefix, prefix_len=torch.tensor([100, more], dtype=torch.int32).cuda(), max_prefix=more)
    assert int(status) == 1
    assert bool((out[1:] == 0).all()) and bool(((out.double() - tol[0]).abs() <= tol[2])[:1].all())


def test_nothing_is_appended_past_a_view():
    page, Hkv, d = 16, 2, 64
    table = torch.tensor([[0, 1], [2, 3], [4, 5]], dtype=torch.int32)
    t = torch.bfloat16
    pool = torch.full((8, Hkv, page, d), 3.0, dtype=t, device="cuda")
    q, k, v = (torch.full((3, n), 1.0, dtype=t, device="cuda") for n in (Hkv * d, Hkv * d, Hkv * d))
    r = D.make_rotation(Hkv, Hkv, d, D.DART_BF16, torch.ones(32, device="cuda"))
    pos = torch.zeros(3, dtype=torch.int64, device="cuda")
    for before, after in ((0, 4), (5, 2), (6, 0)):
        view = inside(table, before, after, [6, 7])  # (pages of nobody)
        for kv, put, bits in (([5, 32, 17], [5, 32, 17], 0), ([5, 33, 17], [5, None, 17], 1), ([40, 1, 64], [None, 1, None], 1)):
            k_pool, v_pool = pool.clone(), pool.clone()
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            cache = D.make_cache(Hkv, k_pool, view, torch.tensor(kv, dtype=torch.int32, device="cuda"), 100)
            D.dart_norm_rotate_append(r, cache, q, k, v, pos, torch.empty_like(q), k_pool, v_pool, status=status)
            torch.cuda.synchronize()
            want = pool.clone()
            for b, x in enumerate(put):
                if x is not None:
                    want[int(table[b, (x - 1) // page]), :, (x - 1) % page] = 1.0
            assert int(status) == bits and torch.equal(k_pool, want) and torch.equal(v_pool, want)


def test_packed_tokens_without_a_bound_on_a_sequence():
    c = A.make([5, 1, 0, 70], [33, 9, 4, 70], 4, 2, 64, 16, "bf16", seed=3)
    k_pool, v_pool = c.k_pool.cuda(), c.v_pool.cuda()
    cache = D.make_cache(4, k_pool, c.table.cuda(), torch.tensor(c.kv, dtype=torch.int32).cuda(), 70, T=c.T, cu_q=c.cu.cuda())
    out, lse = torch.empty((c.T, 256), dtype=c.dtype, device="cuda"), torch.empty((c.T, 4), device="cuda")
    D.dart_attend(cache, A.to_gpu(c.q), k_pool, v_pool, out, D.alloc_attend_workspace(cache), scale=0.125, lse=lse)
    torch.cuda.synchronize()
    A.check(c, (out.cpu().view(c.T, 4, 64), lse.cpu()), scale=0.125)
