"""Grids of kvr_continue_shared, kvr_cache_weigh and kvr_cache_evict over the sizes that kvr.h says are served: no
launch has 2^32 threads or more.  Host code with launcher stubs, on the CPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_13361_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def test_no_launch_has_too_many_threads(tmp_path):
    hipcc = os.path.join(ROCM, "bin", "hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("ROCm compilers not available")
    exe = str(tmp_path / "readers_grids")
    srcs = [os.path.join(CSRC, "kvr_api.hip"), os.path.join(CSRC, "readers", "readers_api.hip"),
            os.path.join(ROOT, "tests", "sanitize", "readers_grids_driver.cpp")]
    subprocess.run([hipcc, "-x", "hip", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
                    "-packed-fp32-ops", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC] + srcs + ["-o", exe],
                   check=True, capture_output=True)
    p = subprocess.run([exe], capture_output=True, timeout=300)
    out = p.stdout.decode(errors="replace") + p.stderr.decode(errors="replace")
    assert p.returncode == 0 and "all checks passed" in out, out[:2000]
