"""more_odd's checks on the GPU."""
import pytest

import more_gpu as G
import more_odd

pytestmark = pytest.mark.gpu


def test_bad_pages_of_evicted_keys():
    more_odd.bad_pages_of_evicted_keys(G.evict)
