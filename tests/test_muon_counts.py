"""The matrix optimizer's counts of arrived parts (host code), on the CPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")
def test_a_count_has_one_number_of_parts(tmp_path):
    import __graft_entry__ as ge
    lb = ge._load_by_path("_arc_lib_build_muon_counts", "paper_2510_26709_amd/build.py")
    csrc = os.path.join(ROOT, "paper_2510_26709_amd", "csrc")
    exe = str(tmp_path / "muon_counts_check")
    subprocess.run(["hipcc", *lb.HIP_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", csrc, "-x",
                    "hip", os.path.join(csrc, "arc_muon.hip"),
                    os.path.join(ROOT, "tests", "muon_counts_check.cpp"), "-o", exe], check=True,
                   capture_output=True, timeout=600)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout + r.stderr
