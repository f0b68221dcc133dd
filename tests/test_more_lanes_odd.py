"""more_odd's checks over the kernels' sources on the CPU between guard pages (lanes_more_util), each in a process of its own."""
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path[:0] = [HERE, os.path.dirname(HERE)]

CHECKS = {"bad_pages_of_evicted_keys": "evict", "scales_that_no_append_writes_read": "read",
          "scales_that_no_append_writes_attend": "attend", "weights_of_many_rows": "weights",
          "weights_of_prefixes_of_many_rows": "weights"}


@pytest.mark.parametrize("check", sorted(CHECKS))
def test_out_of_the_ordinary(check):
    import lanes_more_util
    lanes_more_util.build()
    r = subprocess.run([sys.executable, os.path.abspath(__file__), check], capture_output=True, text=True, timeout=900)
    assert r.returncode == 0 and r.stdout.endswith("lanes ok\n"), (r.returncode, r.stdout[-500:], r.stderr[-3000:])


if __name__ == "__main__":
    import torch

    import lanes_more_util as M
    import more_odd

    torch.set_num_threads(1)
    call, how = getattr(M, CHECKS[sys.argv[1]]), dict(packed=True) if CHECKS[sys.argv[1]] == "evict" else {}
    getattr(more_odd, sys.argv[1])(lambda *a, **k: call(*a, **how, **k))
    print("lanes ok", flush=True)
