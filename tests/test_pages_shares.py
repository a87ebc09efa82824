"""How a paged attention call's work is divided (host logic, no GPU): shares of equal length
over tiles of any, each tile's rows covered once and in order, cuts at whole 64 rows."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_29913_amd", "csrc")


def test_shares_cover_the_work_once(tmp_path):
    exe = str(tmp_path / "pages_check")
    cmd = ["g++", "-O2", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", CSRC, "-I",
           os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "pages_check.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        pytest.fail("could not build the checker:\n" + res.stderr[-3000:])
    res = subprocess.run([exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout
    ok, calls, tiles, split = res.stdout.split()
    assert ok == "ok" and int(calls) == 3000 and int(tiles) > 10000 and int(split) > 1000
