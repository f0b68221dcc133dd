"""Counted memory traffic that the benchmark quotes: it belongs to the sources of the step's kernels, and to no others."""
import os
import shutil

import pytest

import bench


@pytest.fixture
def copy(tmp_path, monkeypatch):
    """The benchmark on a copy of the sources and profiles."""
    shutil.copytree(os.path.join(bench.ROOT, "paper_2502_11494_amd", "csrc"), tmp_path / "paper_2502_11494_amd" / "csrc")
    shutil.copytree(os.path.join(bench.ROOT, "profiles"), tmp_path / "profiles")
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return tmp_path / "paper_2502_11494_amd" / "csrc"


def every():
    return [bench.measured_traffic(prefix, config) for config in bench.TRAFFIC_FILES for prefix in ("", "k_row_l1", "k_scores")]


def test_the_committed_counters_are_those_of_the_present_kernels():
    assert all(isinstance(x, int) and x > 0 for x in every())


def test_the_sources_are_the_units_that_the_step_is_built_from():
    names = [os.path.basename(p) for p in bench.step_sources()]
    assert "dart_api.hip" in names and "k_scores.hpp" in names and "pivot_rank.hpp" in names and names == sorted(names)
    assert not {"attend_api.hip", "k_attend.hpp", "k_rotate.hpp", "cache.hpp"} & set(names)


def test_counters_fall_away_with_a_kernel_of_the_step_and_with_no_other(copy):
    want = every()
    with open(copy / "k_attend.hpp", "a") as f:
        f.write("// changed\n")
    (copy / "new.hpp").write_text("// a file that the step does not include\n")
    assert every() == want
    with open(copy / "k_select.hpp", "a") as f:
        f.write("// changed\n")
    assert every() == [None] * len(want)
