"""The rules by which the upkeep of the bf16 cache is launched (no GPU)."""
import os
import shutil
import subprocess

import paper_2601_11822_amd as rs


def test_rules_are_as_measured(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "host_upkeep_check.hip")
    exe, lib = str(tmp_path / "host_upkeep_check"), os.path.dirname(rs.LIB_PATH)
    rs.load()
    subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-std=c++17", src, "-L" + lib, "-l:" + os.path.basename(rs.LIB_PATH), "-Wl,-rpath," + lib, "-o", exe],
                   check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
