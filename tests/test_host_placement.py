"""The cost by which gacer_place_streams ranks tenants knows products of 8-bit rows (tests/sanitize/placement_driver.cpp, host code under sanitizers, no GPU)."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2304_11745_amd", "csrc")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not on PATH")
def test_tenants_are_ranked_by_their_products(tmp_path):
    exe = str(tmp_path / "placement_driver")
    cmd = ["hipcc", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Xarch_host", "-fsanitize=address,undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
           "-x", "hip", os.path.join(CSRC, "executor.cpp"), os.path.join(CSRC, "search.cpp")]
    cmd += [os.path.join(HERE, "sanitize", f) for f in ("stub_kernels.cpp", "stub_hip.cpp", "placement_driver.cpp")] + ["-Wl,--wrap=hipEventElapsedTime", "-o", exe]
    built = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert built.returncode == 0, built.stderr[-4000:]
    ran = subprocess.run([exe], capture_output=True, text=True, timeout=120, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0"))
    assert ran.returncode == 0, (ran.stdout + ran.stderr)[-6000:]
    assert "all checks held" in ran.stdout
