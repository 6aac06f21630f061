"""How kvr_paged_decode shares its work out, the device code itself, compiled for the CPU under sanitizers: 64 contexts
that meet at each operation between lanes stand for a wave.  Every unit once; and lengths that change while the
call runs end a walk inside the batch."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_13361_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def test_units_of_a_batch_on_the_cpu(tmp_path):
    if not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime.h")):
        pytest.skip("ROCm headers not available")
    exe = str(tmp_path / "walk")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-D__HIP_PLATFORM_AMD__",
           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-I" + os.path.join(ROCM, "include"),
           os.path.join(ROOT, "tests", "sanitize", "paged_walk_driver.cpp"), "-o", exe]
    made = subprocess.run(cmd, capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-3000:]
    p = subprocess.run([exe], capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, ASAN_OPTIONS="detect_stack_use_after_return=0:detect_leaks=0"))
    assert p.returncode == 0 and "all checks passed" in p.stdout, (p.stdout + p.stderr)[-3000:]
