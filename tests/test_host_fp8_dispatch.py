"""Launchers of the operators on 8-bit rows without a GPU: what they say of their kernels against what the compiler gave them, and which tiles the sizes of the
GPU tests take."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2304_11745_amd import build
from test_host_token_dispatch import HERE, TOOLS, compiled, held  # noqa: F401  (compiled is a fixture)

TILES = ["gemm_fp8_few", "gemm_fp8_64x32", "gemm_fp8_64x64", "gemm_fp8_128x128", "gemm_fp8_256x128", "gated_fp8_256x32", "gated_fp8_256x64", "gated_fp8_256x128"]


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if shutil.which("hipcc") is None or not all(map(os.path.exists, TOOLS)):
        pytest.skip("no compiler or no LLVM tools")
    exe = str(tmp_path_factory.mktemp("driver") / "fp8_dispatch_driver")
    cmd = ["hipcc", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-x", "hip", os.path.join(HERE, "fp8_dispatch_driver.cpp"), "-x", "none", build.LIB, "-Wl,-rpath," + os.path.dirname(build.LIB), "-o", exe]
    built = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert built.returncode == 0, built.stderr[-4000:]
    return exe


def test_launchers_know_their_kernels(driver, compiled):  # noqa: F811
    told = [line.split() for line in subprocess.run([driver], check=True, capture_output=True, text=True, timeout=60).stdout.splitlines()]
    wrong, seen = [], set()
    for name, per_unit, lds, threads in told:
        match = [k for k in compiled if name in k]
        assert len(match) == 1, (name, match)
        registers, bytes_, most = compiled[match[0]]
        seen.add(match[0])
        if (int(per_unit), int(lds), int(threads)) != (held(registers, bytes_, most), bytes_, most):
            wrong.append((name, (per_unit, lds, threads), registers, (held(registers, bytes_, most), bytes_, most)))
    assert not wrong, wrong
    ours = {k for k in compiled if re.search("fp8_", k)}
    assert seen == ours, ours - seen


def test_the_gpu_tests_take_every_tile(driver):
    import test_gpu_fp8 as G
    seen = set()
    for gated, batch, tokens, cin, cout in [(0, *s) for s in G.SHAPES + G.WIDE_GEMMS] + [(1, *s) for s in G.SHAPES + G.WIDE_GATED]:
        out = subprocess.run([driver, str(gated), str(batch * tokens), str(cin), str(-(-cout // 16) * 16 if gated else cout), "codes"][:6 if gated else 5], check=True, capture_output=True, text=True,
                             timeout=60).stdout.split()
        seen.add((out[0].replace("_bf16", ""), int(out[1]) > 1))
    for tile in TILES:
        assert (tile, False) in seen, (tile, sorted(seen))
    for tile in TILES:
        assert (tile, True) in seen, (tile, sorted(seen))
