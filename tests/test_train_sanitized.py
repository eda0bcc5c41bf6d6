"""The host side of the training operators under AddressSanitizer (with leak
checking) on the CPU: its sources, host code instrumented and device code built
as usual, linked with tests/train_asan_check.cpp."""
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")
def test_host_code_under_asan(tmp_path):
    import __graft_entry__ as ge
    lb = ge._load_by_path("_arc_lib_build_train_asan", "paper_2510_26709_amd/build.py")
    csrc = os.path.join(ROOT, "paper_2510_26709_amd", "csrc")
    sources = [os.path.join(csrc, f) for f in ("arc_train.cpp", "arc_tokens.hip",
                                               "arc_optim.hip")]
    sources.append(os.path.join(ROOT, "tests", "train_asan_check.cpp"))

    def compile_one(src):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        subprocess.run(["hipcc", *lb.HIP_FLAGS, "-g", "-Xarch_host", "-fsanitize=address", "-I",
                        os.path.join(ROOT, "include"), "-I", csrc, "-x", "hip", "-c", src, "-o",
                        obj], check=True, capture_output=True, timeout=600)
        return obj

    with ThreadPoolExecutor(4) as pool:
        objs = list(pool.map(compile_one, sources))
    exe = str(tmp_path / "train_asan_check")
    subprocess.run(["hipcc", "--offload-arch=gfx950", *objs, "-Xarch_host", "-fsanitize=address",
                    "-o", exe], check=True, capture_output=True, timeout=300)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0, r.stdout + r.stderr[-4000:]
    assert r.stdout.strip().endswith("ok")
    assert "AddressSanitizer" not in r.stderr, r.stderr[-4000:]
