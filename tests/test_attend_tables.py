"""Page tables that are views of wider ones: what the descriptor says about them."""
import torch

import paper_2502_11494_amd as D

from test_attend_host import BAD_CACHE, FAKE, attend, cache  # noqa: F401


def test_a_view_of_a_table_keeps_its_own_width():
    pool, kv = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16), torch.ones(4, dtype=torch.int32)
    base = torch.zeros((4, 32), dtype=torch.int32)
    c = D.make_cache(4, pool, base[:, 24:32], kv, 128)
    assert (c.pages_ld, c.pages_n) == (32, 8)
    c = D.make_cache(4, pool, base, kv, 128)
    assert (c.pages_ld, c.pages_n) == (32, 32)
    c = D.make_cache(4, pool, base[2:3, 5:9], kv[:1], 128)
    assert c.pages_n == 4 and c.pages_ld >= 1
    front = dict(group_cu=torch.tensor([0, 2, 4], dtype=torch.int32), prefix_len=torch.ones(2, dtype=torch.int32), max_prefix=99)
    c = D.make_cache(4, pool, base[:, 24:32], kv, 128, prefix_pages=base[:2, 3:9], **front)
    assert (c.prefix_ld, c.prefix_n, c.max_prefix) == (32, 6, 99)
    # without columns no key has a page
    c = D.make_cache(4, pool, base[:, 9:9], kv, 128, prefix_pages=base[:2, 3:3], **front)
    assert c.pages_ld >= 1 and c.max_kv == 0 and c.prefix_ld >= 1 and c.max_prefix == 0


def test_widths_of_tables_are_checked_and_default_to_the_stride():
    groups = dict(groups=1, prefix_ld=4, max_prefix=9, group_cu=FAKE, prefix_pages=FAKE, prefix_len=FAKE)
    need = D.dart_attend_workspace_bytes(cache(**groups))
    assert need > 0
    for kw in (dict(pages_n=-1), dict(prefix_n=-1)):
        assert D.dart_attend_workspace_bytes(cache(**groups, **kw)) == 0
        assert attend(cache(**groups, **kw)) == D.DART_ERR_SHAPE
    assert D.dart_attend_workspace_bytes(cache(**groups, pages_n=20, prefix_n=4)) == need
    assert D.dart_attend_workspace_bytes(cache(prefix_n=-1)) > 0  # (without groups their fields are ignored)


def test_packed_tokens_without_a_bound_may_all_be_of_one_sequence():
    pool, pages = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((2, 4), dtype=torch.int32)
    kv, cu = torch.tensor([20, 30], dtype=torch.int32), torch.tensor([0, 2, 9], dtype=torch.int32)
    assert D.make_cache(4, pool, pages, kv, 64, T=9, cu_q=cu).max_q == 9
    assert D.make_cache(4, pool, pages, kv, 64, T=9, max_q=7, cu_q=cu).max_q == 7
    assert D.make_cache(4, pool, pages, kv, 64, T=9, max_q=0, cu_q=cu).max_q == 0
    assert D.make_cache(4, pool, pages, kv, 64).max_q == 1


def test_prefixes_without_a_bound_may_fill_their_pages():
    pool, pages = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((2, 4), dtype=torch.int32)
    kv, ints = torch.tensor([20, 30], dtype=torch.int32), lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    front = dict(group_cu=ints(0, 2), prefix_pages=torch.zeros((1, 9), dtype=torch.int32), prefix_len=ints(100))
    assert D.make_cache(4, pool, pages, kv, 64, **front).max_prefix == 9 * 16
    assert D.make_cache(4, pool, pages, kv, 64, **front, max_prefix=100).max_prefix == 100
    assert D.make_cache(4, pool, pages, kv, 64, **front, max_prefix=0).max_prefix == 0
    assert D.make_cache(4, pool, pages, kv, 64).max_prefix == 0
