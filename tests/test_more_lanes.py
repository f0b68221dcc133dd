"""What the kernels on 4-bit pages, gathered weights and eviction address: their sources on the CPU, every buffer between guard
pages and of exactly the size that the header asks for, over ragged, empty, invalid and padded calls."""
import os
import subprocess
import sys

import pytest

import lanes_more_util

RUN = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lanes_more_run.py")
GROUPS = ("hold", "attend", "share", "weights", "prefixes", "evict", "garbage")


@pytest.fixture(scope="module")
def started(tmp_path_factory):
    """All groups side by side, a thread each."""
    lanes_more_util.build()
    folder = tmp_path_factory.mktemp("lanes")
    runs = {g: subprocess.Popen([sys.executable, RUN, g], stdout=open(folder / f"{g}.out", "w"), stderr=open(folder / f"{g}.err", "w"))
            for g in GROUPS}
    yield runs, folder
    for p in runs.values():
        if p.poll() is None:
            p.kill()
            p.wait()


@pytest.mark.parametrize("group", GROUPS)
def test_no_access_is_out_of_bounds(started, group):
    runs, folder = started
    code = runs[group].wait(timeout=900)
    out, err = (open(folder / f"{group}.{x}").read() for x in ("out", "err"))
    assert code == 0 and out.endswith("lanes ok\n"), (code, out[-500:], err[-3000:])
