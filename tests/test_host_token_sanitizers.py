"""Host code of the operators of a decoding tenant under AddressSanitizer and UndefinedBehaviorSanitizer: tests/sanitize/token_driver.cpp loads, plans,
runs, profiles and searches tenants whose operators have no output or no input tensor, on geometry-only kernels and a HIP runtime made of host code.
The sanitizers apply to host code only."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2304_11745_amd", "csrc")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not on PATH")
def test_a_decoding_tenant_is_walked_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "token_driver")
    cmd = ["hipcc", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Xarch_host", "-fsanitize=address,undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
           "-x", "hip", os.path.join(CSRC, "executor.cpp"), os.path.join(CSRC, "search.cpp")]
    cmd += [os.path.join(HERE, "sanitize", f) for f in ("stub_kernels.cpp", "stub_hip.cpp", "token_kernels.cpp", "token_driver.cpp")] + ["-Wl,--wrap=hipGetDevice,--wrap=hipSetDevice", "-o", exe]
    built = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert built.returncode == 0, built.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    ran = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert ran.returncode == 0, (ran.stdout + ran.stderr)[-6000:]
    assert "all checks held" in ran.stdout
