"""The host code of the rotation, cache and attention calls (argument checks, the plan of a launch, workspace
arithmetic) under AddressSanitizer and UndefinedBehaviorSanitizer, 60 000 descriptors.  No GPU is involved."""
import os
import subprocess

from paper_2502_11494_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_attend_host_code_is_clean_under_asan_and_ubsan():
    outdir = os.path.join(ROOT, "_build")
    build.build_host_sanitized(outdir)
    exe = os.path.join(outdir, "attend_host_sanitize")
    subprocess.run(["/opt/rocm/llvm/bin/clang", "-O1", "-g", "-Wall", "-Werror", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "attend_host_sanitize.c"), "-L", outdir,
                    "-ldart_hip_san", "-Wl,-rpath," + outdir, "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "sanitize ok" in r.stdout, (r.returncode, r.stdout[-300:], r.stderr[-3000:])
