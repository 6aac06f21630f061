"""AddressSanitizer / UndefinedBehaviorSanitizer build of the host side of
kvr_qk_norm_rope, kvr_paged_append and kvr_paged_decode, run on the CPU: a
deterministic fuzz of descriptors and sizes whose launcher stubs check the plans
(every row of every token once, every unit of work found again in its range,
records within the workspace, grids below 2^32 threads).  Sanitizers are applied to host code only."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = os.path.join(ROOT, "tests", "sanitize")
CSRC = os.path.join(ROOT, "paper_2606_13361_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def test_paged_host_code_under_sanitizers(tmp_path):
    hipcc, clang = os.path.join(ROCM, "bin", "hipcc"), os.path.join(ROCM, "llvm", "bin", "clang++")
    if not (os.path.exists(hipcc) and os.path.exists(clang)):
        pytest.skip("ROCm compilers not available")
    host = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
            "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-omit-frame-pointer"]
    objs = []
    for src in (os.path.join(CSRC, "kvr_api.hip"), os.path.join(CSRC, "paged", "paged_api.hip"),
                os.path.join(SAN, "paged_driver.cpp")):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        subprocess.run([hipcc, "-x", "hip", "-c", "-fPIC", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
                        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"] + host +
                       ["-I" + os.path.join(ROOT, "include"), "-I" + CSRC, src, "-o", obj], check=True, capture_output=True)
        objs.append(obj)
    exe = str(tmp_path / "paged_driver")
    subprocess.run([clang, "-fsanitize=address,undefined"] + objs +
                   ["-L" + os.path.join(ROCM, "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.join(ROCM, "lib"), "-o", exe],
                   check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0:halt_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    p = subprocess.run([exe], env=env, capture_output=True, timeout=600)
    out = p.stdout.decode(errors="replace") + p.stderr.decode(errors="replace")
    assert p.returncode == 0 and "all checks passed" in out, out[-4000:]
    assert "ERROR: AddressSanitizer" not in out and "runtime error:" not in out, out[-4000:]
