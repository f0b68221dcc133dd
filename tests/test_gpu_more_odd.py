"""more_odd's checks on the GPU."""
import pytest

import more_gpu as G
import more_odd

pytestmark = pytest.mark.gpu


def test_bad_pages_of_evicted_keys():
    more_odd.bad_pages_of_evicted_keys(G.evict)


def test_scales_that_no_append_writes():
    more_odd.scales_that_no_append_writes_read(G.read)
    more_odd.scales_that_no_append_writes_attend(G.attend)


def test_weights_of_many_rows():
    more_odd.weights_of_many_rows(G.weights)
    more_odd.weights_of_prefixes_of_many_rows(G.weights)
