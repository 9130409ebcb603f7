"""The argument checks of the root-mean-square norm, matrices in 8 bits and the
softmax loss under the host address and undefined-behaviour sanitizers (CPU
only): tests/sanitize/ops8_driver.cpp calls every entry point with random and extreme descriptors, the launches
replaced by checks of what the kernels rely on."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.timeout(600)
def test_operator_checks_under_sanitizers(tmp_path):
    if not (os.path.exists(HIPCC) and shutil.which("g++")):
        pytest.skip("hipcc or g++ not available")
    exe = str(tmp_path / "ops8_checks")
    srcs = [os.path.join(ROOT, "paper_2510_12494_amd", "csrc", "ops8.cpp"),
            os.path.join(ROOT, "tests", "sanitize", "ops8_driver.cpp")]
    san = []
    for opt in ("-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=all"):
        san += ["-Xarch_host", opt]
    cmd = [HIPCC, "-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", *san, *srcs, "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, cwd=str(tmp_path))
    assert r.returncode == 0, r.stdout + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1", HIP_VISIBLE_DEVICES="")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "operator checks passed" in r.stdout, out[-4000:]
    assert "runtime error" not in out and "AddressSanitizer" not in out, out[-4000:]
