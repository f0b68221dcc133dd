"""What the attention calls accept of the largest sizes that the header names: host checks."""
import pytest

import paper_2502_11494_amd as D

from test_attend_host import FAKE, attend, cache


def plan(**kw):
    return D.dart_attend_workspace_bytes(cache(**kw))


@pytest.mark.parametrize("B,Hkv", [(1 << 20, 8), (1 << 20, 16), (262144, 32), (1 << 20, 256)])
def test_single_tokens_of_many_sequences(B, Hkv):
    """As many blocks as it takes: rows of one part each, so nothing limits the (token, head) pairs but T * Hq/Hkv."""
    one = dict(B=B, T=B, cu_q=None, Hq=Hkv, Hkv=Hkv, d=8, max_q=1, max_kv=64, row_ld=8, head_ld=128, page_ld=128 * Hkv, pages_ld=4)
    assert plan(**one) > 0
    assert plan(**dict(one, cu_q=FAKE)) > 0
    assert attend(cache(**one), q_ld=8 * Hkv, out_ld=8 * Hkv, ws=None) == D.DART_ERR_WORKSPACE  # (all else is accepted)
    assert plan(**dict(one, B=B + (1 << 20), T=B + (1 << 20))) == 0


def test_limits_of_rows_and_of_pairs_that_are_joined():
    many = dict(B=16, T=1 << 24, max_q=1 << 20, max_kv=64, Hkv=1, d=8, row_ld=8, head_ld=128, page_ld=128, pages_ld=4)
    assert plan(**dict(many, Hq=16)) > 0                      # 2^28 rows
    assert plan(**dict(many, Hq=32)) == 0
    front = dict(groups=2, prefix_ld=4, max_prefix=64, group_cu=FAKE, prefix_pages=FAKE, prefix_len=FAKE)
    assert plan(**dict(many, **front, Hq=1)) > 0              # 2^24 pairs in two parts
    assert plan(**dict(many, **front, Hq=2)) == 0
    assert plan(**dict(many, **front, Hq=2, Hkv=2, T=1 << 23)) > 0
