"""The assembly of the attention kernels.  Kernels short of vector registers park some in accumulation registers.  Where a short
branch that only some lanes take is not jumped over, the compiler has put such copies in front of the instruction that lets all
lanes go on: the others then find anything in their place, addresses among them.  No copy may stand there."""
import os
import re
import subprocess

from paper_2502_11494_amd import build

COPY = re.compile(r"v_accvgpr_(write|mov)|scratch_store")


def parked_by_some_lanes(assembly):
    """(kernel, line, instruction) of copies between the start of a block and the restore of the lanes in it."""
    found, kernel, block = [], None, []
    for n, line in enumerate(assembly.splitlines(), 1):
        name = re.match(r"(_Z\w+):", line)
        if name or re.match(r"\.LBB|; %bb", line):
            kernel, block = (name.group(1) if name else kernel), []
            continue
        text = line.split(";")[0].strip()
        if text.startswith("s_or_b64 exec, exec"):
            found += [(kernel, k, t) for k, t in block if COPY.match(t)]
            block = []
        elif text:
            block.append((n, text))
    return found


def test_the_scan_finds_a_copy_before_the_lanes_are_restored():
    bad = "_Zk:\n\ts_and_saveexec_b64 s[0:1], vcc\n; %bb.1:\n\tds_write_b32 v1, v2\n; %bb.2:\n\tv_accvgpr_write_b32 a80, v34\n"
    end = "\ts_or_b64 exec, exec, s[0:1]\n"
    assert parked_by_some_lanes(bad + end) == [("_Zk", 6, "v_accvgpr_write_b32 a80, v34")]
    assert parked_by_some_lanes(bad.replace("; %bb.2:\n", "; %bb.2:\n" + end)) == []


def test_no_register_is_parked_by_some_lanes_only(tmp_path):
    out = tmp_path / "attend.s"
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "-S", "--cuda-device-only",
                    os.path.join(build.CSRC, "attend_api.hip"), "-o", str(out)], check=True, capture_output=True)
    assembly = out.read_text()
    assert assembly.count("s_or_b64 exec, exec") > 100
    assert parked_by_some_lanes(assembly) == []
