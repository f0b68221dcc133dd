"""The assembly of the kernels on 4-bit pages, gathered weights and eviction, read as test_device_code reads that of the
attention kernels; and no kernel of theirs spills registers to memory."""
import os
import re
import subprocess

import pytest

from paper_2502_11494_amd import build
from test_device_code import parked_by_some_lanes


@pytest.mark.parametrize("unit", ["fourbit_api", "evict_api"])
def test_no_register_is_parked_by_some_lanes_only_and_none_in_memory(tmp_path, unit):
    out = tmp_path / "unit.s"
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "-S", "--cuda-device-only",
                    os.path.join(build.CSRC, unit + ".hip"), "-o", str(out)], check=True, capture_output=True)
    assembly = out.read_text()
    assert assembly.count("s_or_b64 exec, exec") > 100
    assert parked_by_some_lanes(assembly) == []
    kernels = re.findall(r"\.name:\s+(_Z\w+)\n(?:.*\n)*?\s+\.private_segment_fixed_size: (\d+)", assembly)
    assert len(kernels) > 20
    assert [k for k, n in kernels if int(n) > 0] == []
