"""What the rotation and attention kernels address: their sources on the CPU, every buffer between guard pages and of exactly the
size that the header asks for, over ragged, empty, invalid and padded calls in every kind of tile."""
import os
import subprocess
import sys

import pytest

import lanes_util

RUN = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lanes_run.py")
GROUPS = ("tiles", "widest", "prefixes", "joins", "garbage", "rows")


@pytest.fixture(scope="module")
def started(tmp_path_factory):
    """All groups side by side, a thread each."""
    lanes_util.build()
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


def test_an_access_out_of_bounds_does_end_the_process():
    """A page table a row short of what its descriptor says (on the CPU, of course)."""
    lanes_util.build()
    code = (f"import sys; sys.path[:0] = [{os.path.dirname(RUN)!r}, {lanes_util.ROOT!r}]\n"
            "import attend_util as A, lanes_util as L\n"
            "c = A.make([1, 1], [40, 40], 2, 1, 64, 16, 'bf16')\n"
            "c.table = c.table[:1]\n"
            "L.attend(c, scale=0.1)\nprint('went unnoticed')\n")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode < 0 and "went unnoticed" not in r.stdout, (r.returncode, r.stdout, r.stderr[-2000:])
